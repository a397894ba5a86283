// Softmax cross entropy of rows against many classes, without keeping the logits: loss and gradients.
//
//   z = scale * X W^T + bias;  lse_n = log sum_v exp z_nv;  loss_n = lse_n - z_n,label
//   d = dloss_n (softmax(z) - [v = label]);  dbias = sum_n d;  dX = scale d W;  dW = scale d^T X
//
// All of it is products of three forms on tiles that go through LDS, and what happens to a tile's sums at its end:
//   logits     X W^T  : both operands lie along k; the end takes the largest and the sum of exponentials of the tile's
//                       part of a row, or forms d in 16 bits, for a piece of the classes at a time
//   rows' gradient    d W : the second operand lies across k
//   classes' gradient d^T X : both do
// What lies across k is read from LDS by ds_read_b64_tr_b16, which gives a lane four elements from four of LDS's rows, so that
// nothing is transposed in memory.
// 16-bit rows use the 16-bit matrix instructions, sums in 32 bits; d is rounded to the rows' type like any operand of theirs (for
// fp16 times a power of two that brings the largest dloss to 2^14, where no probability that counts is lost).  With the
// result's own rounding that leaves gradients off by 1.4 times what the result's alone would (2.4e-3 against 1.7e-3 of the norm in bf16,
// 2.9e-4 against 2.1e-4 in fp16); a second piece of d would double the gradients' products.
// 32-bit rows are split into three bf16 pieces each (24 bits), of whose products the six largest are
// added: what is left out is below 2^-24 of the magnitudes.
#include <math.h>

#include "ftk_mma.h"
#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint16_t half8 __attribute__((ext_vector_type(8)));

constexpr int XENT_STAGE = 64;  // elements of k in LDS at a time: a line of 128 bytes
constexpr int64_t XENT_MAX_LD = 1 << 23;  // elements of a row: offsets within a tile are 32 bits wide
constexpr int XENT_MAX_D = 1 << 20;

// One operand: `outer` rows or columns of the result by `inner` elements of k.
// Along k: rows of ld elements.  Across k: rows are k.  Multiples of eight elements, 16-byte aligned.
struct Operand {
    const uint16_t *p;
    int64_t ld, plane;  // elements from one bf16 piece of the rows to the next
    int64_t outer, inner;
};
struct Product {
    Operand a, b;  // the result's rows and columns
    uint32_t mt, nt;  // tiles
    int stages;  // of k
    int splits;  // workgroups that share a tile's stages out between them
};

template <int MT_, int NT_, int WM_, int WN_>
struct Shape {
    static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = 16 * MT * WM, TN = 16 * NT * WN;
    static constexpr int A = TM * 128, STAGE = (TM + TN) * 128, LDS = 2 * STAGE;
    // of 32 elements of three pieces
    static constexpr int A3 = TM * 64, B3 = TN * 64, STAGE3 = 3 * (A3 + B3), LDS3 = 3 * STAGE3;
};

// What a workgroup's end knows of its place.
struct Place {
    int64_t m0, n0;  // of the tile
    int wm, wn;      // of the wave within it
    uint32_t mtile, ntile;
    int split;
};

// Row of row tile i, and column of column tile j, that lane row r (of 16) has.  Two column tiles give a lane eight consecutive
// columns of a result row; what lies across k is read the same way.
template <bool ACROSS>
__device__ __forceinline__ int line_of(int i, int r)
{
    return ACROSS ? 32 * (i >> 1) + 8 * (r >> 2) + 4 * (i & 1) + (r & 3) : 16 * i + r;
}

// Pieces of 16 bytes are stored at their place xor a key, so that lanes that read together meet all banks.
// Along k: the rows that 16 lanes read differ in the key or in their place among 256 bytes (lines of 8 pieces, or of 4).
template <bool PERMUTED, int K>
__device__ __forceinline__ int line_key(int row)
{
    if (K == 32) {  // (of four rows: 0, 2, 3, 1; quarters of 64 lanes are read crosswise)
        const int x = row >> (PERMUTED ? 3 : 2);
        return (x >> 1 & 1) | ((x ^ x >> 1) & 1) << 1;
    }
    return PERMUTED ? ((row >> 1) & 1) | ((row >> 3) & 3) << 1 : (row >> 1) & 7;
}
// Across k (T columns, T / 8 pieces a row): four rows of k, four pieces each.
template <int T>
__device__ __forceinline__ int across_key(int k)
{
    return T >= 128 ? (k & 3) * 4 : (k >> 1 & 1) * 4;
}

// Copies of one operand's tile of T rows (columns) by K elements of k to LDS, a share of them a wave.
template <int T, int WAVES, bool ACROSS, bool PERMUTED, int K>
struct Copies {
    static constexpr int N = T * K / 512 / WAVES;  // of a wave
    static constexpr int LINE = K / 8;             // pieces of a line along k
    uint32_t off[N];
    const uint8_t *base;
    int64_t step;  // bytes of a stage
    static __device__ __forceinline__ int k_of(int c, int lane) { return c * (512 / T) + lane / (T / 8); }
    static __device__ __forceinline__ int piece_of(int c, int lane)
    {
        if (ACROSS) return (lane & (T / 8 - 1)) ^ across_key<T>(k_of(c, lane));
        return (lane & (LINE - 1)) ^ line_key<PERMUTED, K>(row_of(c, lane));
    }
    static __device__ __forceinline__ int row_of(int c, int lane) { return c * (64 / LINE) + lane / LINE; }
    __device__ __forceinline__ void begin(const Operand &o, int64_t first, int w, int lane)
    {
        base = (const uint8_t *)(o.p + (ACROSS ? first : first * o.ld));
        step = ACROSS ? K * o.ld * 2 : K * 2;
        const int64_t left = o.outer - first;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = w * N + i;
            int piece = piece_of(c, lane);
            if (ACROSS) {
                if (piece * 8 >= left) piece = 0;
                off[i] = (uint32_t)k_of(c, lane) * (uint32_t)o.ld * 2 + piece * 16;
            } else {
                const int64_t row = row_of(c, lane);
                off[i] = (uint32_t)(row < left ? row : left - 1) * (uint32_t)o.ld * 2 + piece * 16;
            }
        }
    }
    // where stage st begins, of piece `plane` of the rows
    __device__ __forceinline__ const uint8_t *from(const Operand &o, int plane, int st) const
    {
        return uniform(base + plane * o.plane * 2 + st * step);
    }
    // copy i of a stage, of whose elements of k `left` are left
    __device__ __forceinline__ void copy(const Operand &o, const uint8_t *stage, int left, uint32_t lds, int w, int lane, int i) const
    {
        const int c = w * N + i;
        uint32_t at = off[i];
        if (left < K) {
            asm volatile("");  // (a branch that is hardly ever taken, rather than its arithmetic every time)
            if (ACROSS) {
                const int k = k_of(c, lane);
                if (k >= left) at -= (uint32_t)(k - left + 1) * (uint32_t)o.ld * 2;
            } else if (piece_of(c, lane) * 8 >= left) {
                at -= piece_of(c, lane) * 16;
            }
        }
        to_lds16_from(stage, at, lds + c * 1024);
    }
};

// Fragments of one operand: 16 rows (columns), lane quarter q has elements 8 q ... of a step of 32.
template <int T, bool ACROSS, bool PERMUTED, int K>
struct Fragments {
    // first: of the wave's rows within the tile
    static __device__ __forceinline__ half8 read(const uint8_t *lds, int first, int i, int s, int lane)
    {
        const int r = lane & 15, q = lane >> 4;
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) short4v lds4;
            const int k = s * 32 + q * 8 + (r >> 2), piece = (first >> 3) + 4 * (i >> 1) + (r & 3);
            const uint8_t *p = lds + k * (T * 2) + (piece ^ across_key<T>(k)) * 16 + (i & 1) * 8;
            // (k + 4 has the same key)
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p);
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 4 * T * 2));
            return __builtin_bit_cast(half8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int row = first + line_of<PERMUTED>(i, r);
            return *reinterpret_cast<const half8 *>(lds + row * (K * 2) + ((s * 4 + q) ^ line_key<PERMUTED, K>(row)) * 16);
        }
    }
};

template <typename H>
__device__ __forceinline__ float4v mma(half8 b, half8 a, float4v c)
{
    typedef H vec __attribute__((ext_vector_type(8)));
    if constexpr (std::is_same<H, __bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(vec, b), __builtin_bit_cast(vec, a), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(vec, b), __builtin_bit_cast(vec, a), c, 0, 0, 0);
}

// Workgroups are dealt to the eight XCDs in turn; each XCD gets a run of tiles, eight rows of tiles high, so that the 32 tiles
// under way there share their operands in its L2.  Shares of the stages come one after the other: those of one share read the same.
template <typename S>
__device__ __forceinline__ Place place_of(const Product &g, int w)
{
    const uint32_t tiles = g.mt * g.nt, all = tiles * g.splits, each = (all + 7) / 8;
    const uint32_t x = blockIdx.x & 7, full = all & 7;  // the first `full` XCDs have one more where all is no multiple
    uint32_t t = full ? x * (each - 1) + min(x, full) + (blockIdx.x >> 3) : x * each + (blockIdx.x >> 3);
    Place at;
    at.split = g.splits > 1 ? (int)(t / tiles) : 0;
    t -= at.split * tiles;
    const uint32_t panel = t / (8 * g.nt), in = t - panel * 8 * g.nt, high = min(8u, g.mt - panel * 8);
    at.ntile = in / high;
    at.mtile = panel * 8 + (in - at.ntile * high);
    at.m0 = (int64_t)at.mtile * S::TM;
    at.n0 = (int64_t)at.ntile * S::TN;
    at.wm = w / S::WN * 16 * S::MT;
    at.wn = w % S::WN * 16 * S::NT;
    return at;
}

// A workgroup's share of the stages.
struct Run {
    int first, stages;
};
__device__ __forceinline__ Run run_of(const Product &g, int split)
{
    if (g.splits == 1) return Run{0, g.stages};
    const int first = (int)((uint64_t)g.stages * split / (uint32_t)g.splits);
    return Run{first, (int)((uint64_t)g.stages * (split + 1) / (uint32_t)g.splits) - first};
}

// 16-bit rows.  Stages of 64 elements of k, two in LDS, copied there without passing through registers.  Tiles of 256 x 256 by
// eight waves need 128 KB of LDS, of which 64 KB pass for 8.4 MF: matrix instructions are the bound, with what a tile's begin
// and end take (10 and 5 of 47 us at 32 stages), when none are issued.  8192 rows x 65536 classes x 2048, bf16: the sums 1716 to
// 1775 us, 1.24 to 1.28 PF; d and its store in 16 bits 1860 to 1957; rows' and classes' gradient 1680 to 1736 each, up to 1.31 PF.
// The instruction alone, fed from registers, reaches 1.95 PF on such numbers, a library's large product 1.40 to 1.48.  Slower: five
// stages of 32 in a ring (by 20 %), workgroups that go on to further tiles (26 %), four waves of 128 x 128 (45 %), tiles of
// 128 x 128 (30 %), the 32 x 32 x 16 instruction (its own rate is 10 % less).
template <typename S, typename H, bool AT, bool BT, typename End>
__global__ __launch_bounds__(S::THREADS, 2) void product_kernel(Product g, End end)
{
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of<S>(g, w);
    float4v acc[S::MT][S::NT];
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
        for (int j = 0; j < S::NT; ++j) acc[i][j] = float4v{0, 0, 0, 0};
    Copies<S::TM, S::WAVES, AT, false, XENT_STAGE> ca;
    Copies<S::TN, S::WAVES, BT, true, XENT_STAGE> cb;
    ca.begin(g.a, at.m0, w, lane);
    cb.begin(g.b, at.n0, w, lane);
    const Run run = run_of(g, at.split);
    const int total = run.stages;
    constexpr int COPIES = ca.N + cb.N;
    // of the next copy
    const uint8_t *from_a = ca.from(g.a, 0, run.first), *from_b = cb.from(g.b, 0, run.first);
    int left_a = (int)(g.a.inner - (int64_t)run.first * XENT_STAGE), left_b = (int)(g.b.inner - (int64_t)run.first * XENT_STAGE);
    auto copy = [&](int buffer, int c) __attribute__((always_inline)) {
        const uint32_t to = lds0 + buffer * S::STAGE;
        if (c < ca.N) ca.copy(g.a, from_a, left_a, to, w, lane, c);
        else cb.copy(g.b, from_b, left_b, to + S::A, w, lane, c - ca.N);
    };
    auto copied = [&]() __attribute__((always_inline)) {
        from_a += ca.step;
        from_b += cb.step;
        left_a -= XENT_STAGE;
        left_b -= XENT_STAGE;
    };
    half8 a[S::MT], b[2][S::NT];
    auto read_a = [&](int n, int s, int i) __attribute__((always_inline)) {
        a[i] = Fragments<S::TM, AT, false, XENT_STAGE>::read(lds + (n & 1) * S::STAGE, at.wm, i, s, lane);
    };
    auto read_b = [&](int n, int s, int j) __attribute__((always_inline)) {
        b[s][j] = Fragments<S::TN, BT, true, XENT_STAGE>::read(lds + (n & 1) * S::STAGE + S::A, at.wn, j, s, lane);
    };
    // One step's products, row tile by row tile.  Behind each the next step's fragments of that number are read, those of the rows
    // into the registers just used, and those of the columns, which the next step needs first, behind the first ones.  The
    // first step of a stage reads the second one's.  The second step reads the next stage's: after its first row tiles all waves
    // meet, when what the first step read has long come, this stage's place is free for the one after the next, and the
    // next one has arrived.
    constexpr int MEET = S::MT / 8;
    auto step = [&](auto which, auto reads, auto copies, int n) __attribute__((always_inline)) {
        constexpr int s = decltype(which)::value, next = 1 - s, FROM = s ? MEET : 0;
        constexpr bool READS = decltype(reads)::value, COPY = decltype(copies)::value;
        auto meet = [&]() __attribute__((always_inline)) {
            wait_loads<0>();
            __syncthreads();
        };
        if constexpr (READS && s == 1 && MEET == 0) meet();
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
#pragma unroll
            for (int j = 0; j < S::NT; ++j) acc[i][j] = mma<H>(b[s][j], a[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (READS) {
                if (s == 1 && MEET > 0 && i == MEET - 1) meet();
                constexpr int BEGIN = FROM ? FROM - 1 : 0, GROUPS = S::MT - BEGIN;
                if (i >= BEGIN) {
                    const int g = i - BEGIN;
#pragma unroll
                    for (int k = g == 0 ? 0 : i; k <= i; ++k) read_a(n + s, next, k);
#pragma unroll
                    for (int j = 2 * g; j < 2 * g + 2 && j < S::NT; ++j) read_b(n + s, next, j);
                    if constexpr (COPY) {
#pragma unroll
                        for (int c = g * COPIES / GROUPS; c < (g + 1) * COPIES / GROUPS; ++c) copy(n & 1, c);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    using Zero = std::integral_constant<int, 0>;
    using One = std::integral_constant<int, 1>;
    auto stage = [&](auto more, auto copies, int n) __attribute__((always_inline)) {
        step(Zero{}, One{}, Zero{}, n);
        step(One{}, more, copies, n);
        if constexpr (decltype(copies)::value) copied();
    };
    if (total > 0) {
        for (int n = 0; n < 2 && n < total; ++n) {
#pragma unroll
            for (int c = 0; c < COPIES; ++c) copy(n, c);
            copied();
            if (n == 0) {
                wait_loads<0>();
                __syncthreads();
            }
        }
#pragma unroll
        for (int j = 0; j < S::NT; ++j) read_b(0, 0, j);
#pragma unroll
        for (int i = 0; i < S::MT; ++i) read_a(0, 0, i);
        int n = 0;
        for (; n + 2 < total; ++n) stage(One{}, One{}, n);
        if (n + 1 < total) stage(One{}, Zero{}, n++);
        stage(Zero{}, Zero{}, n);
    }
    __syncthreads();
    end.template run<S, AT>(acc, at, lds);
}

// Rows of three bf16 pieces, all of whole stages: a stage holds 32 elements of all pieces, so that six products are formed of what
// is read once.
// While a stage's products are formed, the next one's fragments come from LDS, the one after that is under way, and the third begins
// to come into the place that this one's fragments have left: one meeting a stage.  777 rows x 10007 classes x 333: the sums 55 us,
// d 63, the rows' and the classes' gradient 38 each (31 GF each by six products, 0.84 PF); matrix instructions are busy for 60 % of
// that, the rest is begin, end and a last round of tiles that does not fill the card.  (One piece's product after the other reads
// LDS twice as often: 63, 70, 56 and 69 us.)
template <typename S, bool AT, bool BT, typename End>
__global__ __launch_bounds__(S::THREADS, 2) void pieces_kernel(Product g, End end)
{
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at = place_of<S>(g, w);
    float4v acc[S::MT][S::NT];
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
        for (int j = 0; j < S::NT; ++j) acc[i][j] = float4v{0, 0, 0, 0};
    constexpr int K = 32;
    Copies<S::TM, S::WAVES, AT, false, K> ca;
    Copies<S::TN, S::WAVES, BT, true, K> cb;
    ca.begin(g.a, at.m0, w, lane);
    cb.begin(g.b, at.n0, w, lane);
    const Run run = run_of(g, at.split);
    constexpr int COPIES = 3 * (ca.N + cb.N), READS = 3 * (S::MT + S::NT);
    // of the next copy
    const uint8_t *from_a[3], *from_b[3];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        from_a[p] = ca.from(g.a, p, run.first);
        from_b[p] = cb.from(g.b, p, run.first);
    }
    auto copy = [&](uint32_t place, int c) __attribute__((always_inline)) {
        const uint32_t to = lds0 + place;
        if (c < 3 * ca.N) ca.copy(g.a, from_a[c / ca.N], K, to + c / ca.N * S::A3, w, lane, c % ca.N);
        else c -= 3 * ca.N, cb.copy(g.b, from_b[c / cb.N], K, to + 3 * S::A3 + c / cb.N * S::B3, w, lane, c % cb.N);
    };
    auto copied = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            from_a[p] += ca.step;
            from_b[p] += cb.step;
        }
    };
    half8 a[2][3][S::MT], b[2][3][S::NT];
    auto read = [&](uint32_t place, int turn, int k) __attribute__((always_inline)) {
        const uint8_t *const from = lds + place;
        if (k < 3 * S::MT) {
            const int p = k / S::MT, i = k % S::MT;
            a[turn][p][i] = Fragments<S::TM, AT, false, K>::read(from + p * S::A3, at.wm, i, 0, lane);
        } else {
            const int p = (k - 3 * S::MT) / S::NT, j = (k - 3 * S::MT) % S::NT;
            b[turn][p][j] = Fragments<S::TN, BT, true, K>::read(from + 3 * S::A3 + p * S::B3, at.wn, j, 0, lane);
        }
    };
    using Zero = std::integral_constant<int, 0>;
    using One = std::integral_constant<int, 1>;
    uint32_t place = 0;  // of this stage
    int left = run.stages;
    auto stage = [&](auto turn, auto full) __attribute__((always_inline)) {
        constexpr int now = decltype(turn)::value;
        const bool copies = decltype(full)::value || left > 3;
        if (decltype(full)::value || left > 2) wait_loads<COPIES>();
        else wait_loads<0>();
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        const uint32_t next = place == 2 * S::STAGE3 ? 0 : place + S::STAGE3;
        // (the small products first)
        constexpr int PA[6] = {2, 1, 0, 1, 0, 0}, PB[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
        for (int s = 0; s < 6; ++s) {
#pragma unroll
            for (int i = 0; i < S::MT; ++i) {
                const int part = s * S::MT + i;
                constexpr int PARTS = 6 * S::MT;
#pragma unroll
                for (int k = part * READS / PARTS; k < (part + 1) * READS / PARTS; ++k) read(next, 1 - now, k);
                if (copies) {
#pragma unroll
                    for (int c = part * COPIES / PARTS; c < (part + 1) * COPIES / PARTS; ++c) copy(place, c);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < S::NT; ++j) acc[i][j] = mma<__bf16>(b[now][PB[s]][j], a[now][PA[s]][i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        copied();
        place = next;
        --left;
    };
    if (left > 0) {
        for (int n = 0; n < 3 && n < left; ++n) {
#pragma unroll
            for (int c = 0; c < COPIES; ++c) copy(n * S::STAGE3, c);
            copied();
        }
        if (left > 2) wait_loads<2 * COPIES>();
        else wait_loads<0>();
        __syncthreads();
#pragma unroll
        for (int k = 0; k < READS; ++k) read(0, 0, k);
        while (left > 4) {
            stage(Zero{}, One{});
            stage(One{}, One{});
        }
        while (left > 1) {
            stage(Zero{}, Zero{});
            stage(One{}, Zero{});
        }
        if (left) stage(Zero{}, Zero{});
    }
    __syncthreads();
    end.template run<S, AT>(acc, at, lds);
}

// ---- ends -----------------------------------------------------------------------------------

constexpr float XENT_LOG2E = 1.44269504f;
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x * XENT_LOG2E); }

struct Logits {
    const float *bias;      // NULL: none
    const int32_t *labels;
    int64_t N;
    int64_t first, last;    // classes of this call: `first` is the products' first one
    int64_t V;
    float scale;
    // (what lies behind the last class of the call is closed)
    __device__ __forceinline__ float bias_of(int64_t v) const { return v >= last ? -__builtin_inff() : bias ? bias[v] : 0.f; }
    // number of the label among the columns from v0 on
    __device__ __forceinline__ int label_from(int32_t label, int64_t v0) const
    {
        return label >= 0 && label < last ? (int)max((int64_t)-1, label - v0) : -1;
    }
};

// The tile's part of a row: its largest logit, the sum of exponentials below it, and the label's logit.
struct SumEnd {
    Logits z;
    float2 *parts;  // [N][tiles]
    int64_t tiles;
    float *label_logit;  // [N]
    template <typename S, bool AT>
    __device__ __forceinline__ void run(float4v (&acc)[S::MT][S::NT], const Place &at, uint8_t *lds) const
    {
        const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
        float2 *const part = reinterpret_cast<float2 *>(lds);  // [WN][TM]
        const int64_t v0 = z.first + at.n0 + at.wn + 8 * q;
        float bias[S::NT][4];
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) bias[j][c] = z.bias_of(v0 + 32 * (j >> 1) + 4 * (j & 1) + c);
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
            const int row = at.wm + line_of<AT>(i, r);
            const int64_t n = at.m0 + row;
            const int rel = z.label_from(n < z.N ? z.labels[n] : -1, v0);
            float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
            for (int j = 0; j < S::NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    acc[i][j][c] = fmaf(z.scale, acc[i][j][c], bias[j][c]);
                    top = fmaxf(top, acc[i][j][c]);
                }
            if (__any(rel >= 0 && rel < 16 * S::NT)) {
#pragma unroll
                for (int j = 0; j < S::NT; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (rel == 32 * (j >> 1) + 4 * (j & 1) + c) z_store(n, acc[i][j][c]);
            }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            // (subtracted before the factor: a part may hold masks of the type's lowest value alone)
            const float shift = top > -__builtin_inff() ? top : 0.f;
#pragma unroll
            for (int j = 0; j < S::NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) sum += exp2_of(acc[i][j][c] - shift);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (q == 0) part[at.wn / (16 * S::NT) * S::TM + row] = float2{top, sum};
        }
        __syncthreads();
        for (int row = threadIdx.x; row < S::TM; row += S::THREADS) {
            const int64_t n = at.m0 + row;
            if (n >= z.N) break;
            float2 p = part[row];
#pragma unroll
            for (int k = 1; k < S::WN; ++k) p = joined(p, part[k * S::TM + row]);
            parts[n * tiles + at.ntile] = p;
        }
    }
    __device__ __forceinline__ void z_store(int64_t n, float x) const { label_logit[n] = x; }
    static __device__ __forceinline__ float2 joined(float2 a, float2 b)
    {
        const float top = fmaxf(a.x, b.x), shift = top > -__builtin_inff() ? top : 0.f;
        return float2{top, a.y * exp2_of(a.x - shift) + b.y * exp2_of(b.x - shift)};
    }
};

// Few rows (up to 16 MT): what takes time is reading W once.  A workgroup's eight waves share D out between them, RUN steps of 32
// each, whose part of the rows stays in registers; W goes from memory straight to registers, 16 / RUN / MT column tiles of 16 classes
// at a time, the next ones requested before these are used.  The waves' sums meet in LDS, where the first waves, one
// for a tile, take the softmax on.  (16 rows, 65536 classes of 2048 bf16, 268 MB: 51 us, 5.2 TB/s; two
// launches' time is the rest of the call's 54.)
template <typename H, int MT, int RUN>
__global__ __launch_bounds__(512, 2) void xent_few_kernel(const H *__restrict__ X, int64_t ldx, const H *__restrict__ W, int64_t ldw, int D,
                                                          SumEnd end)
{
    constexpr int CT = 16 / RUN / MT, WAVES = 8;
    __shared__ float4v part[2][WAVES][CT][MT][64];
    __shared__ float2 last[CT][MT * 16];
    const Logits &z = end.z;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    typedef H piece __attribute__((ext_vector_type(8), aligned(2)));
    half8 x[MT][RUN], b[2][CT][RUN];
    const int k0 = w * RUN * 32 + q * 8;
    auto request = [&](int64_t v0, half8 (&to)[CT][RUN]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const H *row = W + min(v0 + c * 16 + r, z.V - 1) * ldw;
#pragma unroll
            for (int s = 0; s < RUN; ++s) to[c][s] = *reinterpret_cast<const half8 *>(row + (k0 + s * 32 < D ? k0 + s * 32 : 0));
        }
    };
    const int64_t step = (int64_t)gridDim.x * 16 * CT;
    int64_t v0 = (int64_t)blockIdx.x * 16 * CT;
    request(v0, b[0]);
    int64_t label[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t n = 16 * i + r;
        label[i] = n < z.N ? z.labels[n] : -1;
        const bool live = label[i] >= 0 && label[i] < z.V;
#pragma unroll
        for (int s = 0; s < RUN; ++s) {
            const int k = k0 + s * 32;
            x[i][s] = half8{0, 0, 0, 0, 0, 0, 0, 0};
            if (live && k < D) x[i][s] = __builtin_bit_cast(half8, *reinterpret_cast<const piece *>(X + n * ldx + k));
        }
    }
    float2 sum[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sum[i] = float2{-__builtin_inff(), 0.f};
    auto tile = [&](half8 (&now)[CT][RUN], half8 (&next)[CT][RUN], int turn) __attribute__((always_inline)) {
        if (v0 + step < z.V) request(v0 + step, next);
        float4v acc[CT][MT];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                acc[c][i] = float4v{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < RUN; ++s) acc[c][i] = mma<H>(now[c][s], x[i][s], acc[c][i]);
                part[turn][w][c][i][lane] = acc[c][i];
            }
        __syncthreads();
        if (w < CT) {
            const int64_t v = v0 + 16 * w + 4 * q;
            float bias[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = z.bias_of(v + e);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                float4v a = part[turn][0][w][i][lane];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) a += part[turn][k][w][i][lane];
                float top = sum[i].x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a[e] = fmaf(z.scale, a[e], bias[e]);
                    if (v + e == label[i] && v + e < z.V) end.z_store(16 * i + r, a[e]);
                    top = fmaxf(top, a[e]);
                }
                const float shift = top > -__builtin_inff() ? top : 0.f;
                float t = sum[i].y * exp2_of(sum[i].x - shift);
#pragma unroll
                for (int e = 0; e < 4; ++e) t += exp2_of(a[e] - shift);
                sum[i] = float2{top, t};
            }
        }
        v0 += step;
    };
    while (v0 < z.V) {
        tile(b[0], b[1], 0);
        if (v0 < z.V) tile(b[1], b[0], 1);
    }
    if (w < CT) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int d = 16; d < 64; d *= 2)
                sum[i] = SumEnd::joined(sum[i], float2{__shfl_xor(sum[i].x, d, 64), __shfl_xor(sum[i].y, d, 64)});
            if (q == 0) last[w][16 * i + r] = sum[i];
        }
    }
    __syncthreads();
    const int n = threadIdx.x;
    if (n >= 16 * MT || n >= z.N) return;
    float2 p = last[0][n];
#pragma unroll
    for (int c = 1; c < CT; ++c) p = SumEnd::joined(p, last[c][n]);
    end.parts[n * end.tiles + blockIdx.x] = p;
}

// L lanes a row: its parts together, with those of earlier pieces of the classes (running, NULL: there are no other pieces).
template <int L>
__global__ __launch_bounds__(256) void xent_loss_kernel(const float2 *parts, int64_t tiles, float2 *running, bool first, bool end,
                                                        const float *label_logit, const int32_t *labels, int64_t N, int64_t V,
                                                        float *loss, float *lse)
{
    const int lane = threadIdx.x & (L - 1);
    const int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L, n = min(row, N - 1);
    float2 sum{-__builtin_inff(), 0.f};
#pragma unroll 4
    for (int64_t t = lane; t < tiles; t += L) sum = SumEnd::joined(sum, parts[n * tiles + t]);
#pragma unroll
    for (int d = 1; d < L; d *= 2) sum = SumEnd::joined(sum, float2{__shfl_xor(sum.x, d, 64), __shfl_xor(sum.y, d, 64)});
    if (lane || row >= N) return;
    if (running) {
        if (!first) sum = SumEnd::joined(running[n], sum);
        if (!end) {
            running[n] = sum;
            return;
        }
    }
    const int64_t label = labels[n];
    const bool live = label >= 0 && label < V;
    const float l = sum.y == 0.f ? -__builtin_inff() : (sum.x > -__builtin_inff() ? sum.x : 0.f) + logf(sum.y);
    lse[n] = live ? l : 0.f;
    loss[n] = live ? l - label_logit[n] : 0.f;
}

// Power of two that brings the largest |dloss| to [2^14, 2^15) (fp16 rows), else 1.
__device__ __forceinline__ float factor_of(const uint32_t *top)
{
    if (!top) return 1.f;
    const int e = (int)(*top >> 23);
    return *top == 0 || e == 255 ? 1.f : __uint_as_float((uint32_t)min(254, max(1, 268 - e)) << 23);
}

// What a row's part of d takes: d_v = weight (exp(z_v - shift) - [v = label] sum).  shift is lse and sum 1, where that is exact enough
// (terms_kernel); a row that is ignored, or all of whose logits are -infinity, has no weight and no label.
struct __align__(16) RowTerms {
    float shift, sum, weight;
    int32_t label;
};

// d of a tile, in 16 bits (or three bf16 pieces), zero in rows and columns that only fill up; sums over the tile's rows.
template <typename H, int PLANES>
struct GradEnd {
    Logits z;
    const RowTerms *terms;  // [rows]
    const uint32_t *top;
    uint16_t *d;        // [rows][ld]
    int64_t ld, plane, rows;
    float *dbias;       // [row tiles][ld], or NULL
    template <typename S, bool AT>
    __device__ __forceinline__ void run(float4v (&acc)[S::MT][S::NT], const Place &at, uint8_t *lds) const
    {
        const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
        const int64_t v0 = z.first + at.n0 + at.wn + 8 * q;
        const float factor = factor_of(top);
        float bias[S::NT][4], sum[S::NT][4];
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                bias[j][c] = z.bias_of(v0 + 32 * (j >> 1) + 4 * (j & 1) + c);
                sum[j][c] = 0.f;
            }
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
            const int64_t n = at.m0 + at.wm + line_of<AT>(i, r);
            const RowTerms row = n < rows ? terms[n] : RowTerms{__builtin_inff(), 0.f, 0.f, -1};
            const float shift = row.shift, g = row.weight * factor;
            const int rel = z.label_from(row.label, v0);
#pragma unroll
            for (int j = 0; j < S::NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    acc[i][j][c] = exp2_of(fmaf(z.scale, acc[i][j][c], bias[j][c]) - shift);
            if (__any(rel >= 0 && rel < 16 * S::NT)) {
#pragma unroll
                for (int j = 0; j < S::NT; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (rel == 32 * (j >> 1) + 4 * (j & 1) + c) acc[i][j][c] -= row.sum;
            }
#pragma unroll
            for (int j = 0; j < S::NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    acc[i][j][c] *= g;
                    sum[j][c] += acc[i][j][c];
                }
            if (n >= rows) continue;
            uint16_t *const to = d + n * ld + at.n0 + at.wn + 8 * q;
#pragma unroll
            for (int j = 0; j < S::NT; j += 2) {
                half8 o[PLANES];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    float x = acc[i][j + (c >> 2)][c & 3];
#pragma unroll
                    for (int k = 0; k < PLANES; ++k) {
                        const H h = (H)x;
                        o[k][c] = __builtin_bit_cast(uint16_t, h);
                        x -= (float)h;
                    }
                }
#pragma unroll
                for (int k = 0; k < PLANES; ++k) *reinterpret_cast<half8 *>(to + k * plane + 16 * j) = o[k];
            }
        }
        if (!dbias) return;
        float *const part = reinterpret_cast<float *>(lds);  // [WM][TN]
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float s = group_sum<16>(sum[j][c]) / factor;
                if (r == 0) part[at.wm / (16 * S::MT) * S::TN + at.wn + 32 * (j >> 1) + 8 * q + 4 * (j & 1) + c] = s;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < S::TN; c += S::THREADS) {
            float s = part[c];
#pragma unroll
            for (int k = 1; k < S::WM; ++k) s += part[k * S::TN + c];
            dbias[at.mtile * ld + at.n0 + c] = s;
        }
    }
};

// The bias' gradient from the sums of all row tiles: 16 classes a workgroup, a sixteenth of the tiles 16 lanes.
struct BiasJob {
    const float *parts;  // [tiles][ld]
    int64_t ld;
    int tiles;
    int64_t n;
    float *out;
    __device__ __forceinline__ void run(uint32_t group) const
    {
        __shared__ double sums[16][16];
        const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
        const int64_t v = (int64_t)group * 16 + lane;
        double s = 0;
        if (v < n) {
#pragma unroll 8
            for (int t = share; t < tiles; t += 16) s += parts[t * ld + v];
        }
        sums[share][lane] = s;
        __syncthreads();
        if (share || v >= n) return;
        for (int i = 1; i < 16; ++i) s += sums[i][lane];
        out[v] = (float)s;
    }
};
__global__ __launch_bounds__(256) void dbias_kernel(BiasJob job) { job.run(blockIdx.x); }

// A gradient: the sums times `scale` (and what d was multiplied by taken out), added to those of earlier pieces of the classes.
template <typename T>
struct StoreEnd {
    T *out;
    int64_t ld, rows, cols;
    float *sums;  // of earlier and later pieces, or NULL
    int64_t lds;  // a row of theirs
    bool first, last;
    float scale;
    const uint32_t *top;
    template <typename S, bool AT>
    __device__ __forceinline__ void run(float4v (&acc)[S::MT][S::NT], const Place &at, uint8_t *) const
    {
        const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
        const float f = scale / factor_of(top);
        typedef T Eight __attribute__((ext_vector_type(8), aligned(sizeof(T))));
        typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < S::MT; ++i) {
            const int64_t m = at.m0 + at.wm + line_of<AT>(i, r);
            if (m >= rows) continue;
#pragma unroll
            for (int j = 0; j < S::NT; j += 2) {
                const int64_t n = at.n0 + at.wn + 16 * j + 8 * q;
                if (n >= cols) continue;
                float v[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) v[c] = acc[i][j + (c >> 2)][c & 3];
                const bool whole = n + 8 <= cols;
                if (sums) {
                    float *const s = sums + m * lds + n;
                    if (!first) {
#pragma unroll
                        for (int c = 0; c < 8; c += 4) {
                            if (whole) {
                                const Four x = *reinterpret_cast<const Four *>(s + c);
#pragma unroll
                                for (int k = 0; k < 4; ++k) v[c + k] += x[k];
                            } else {
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (n + c + k < cols) v[c + k] += s[c + k];
                            }
                        }
                    }
                    if (!last) {
#pragma unroll
                        for (int c = 0; c < 8; c += 4) {
                            if (whole) {
                                *reinterpret_cast<Four *>(s + c) = Four{v[c], v[c + 1], v[c + 2], v[c + 3]};
                            } else {
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (n + c + k < cols) s[c + k] = v[c + k];
                            }
                        }
                        continue;
                    }
                }
                T *const o = out + m * ld + n;
                if (whole) {
                    Eight x;
#pragma unroll
                    for (int c = 0; c < 8; ++c) x[c] = (T)(v[c] * f);
                    *reinterpret_cast<Eight *>(o) = x;
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (n + c < cols) o[c] = (T)(v[c] * f);
                }
            }
        }
    }
};

// Sums of a share of the stages, [splits][rows][cols].
struct PartEnd {
    float *parts;
    int64_t rows, cols;
    template <typename S, bool AT>
    __device__ __forceinline__ void run(float4v (&acc)[S::MT][S::NT], const Place &at, uint8_t *lds) const
    {
        StoreEnd<float>{parts + at.split * rows * cols, cols, rows, cols, nullptr, 0, true, true, 1.f, nullptr}.template run<S, AT>(acc, at, lds);
    }
};
// All shares together, and what StoreEnd does; workgroups behind those: the bias' gradient.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ parts, int splits, StoreEnd<T> end, uint32_t groups, BiasJob bias)
{
    if (blockIdx.x >= groups) return bias.run(blockIdx.x - groups);
    const int64_t all = end.rows * end.cols;
    const float f = end.scale / factor_of(end.top);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)groups * 256) {
        float s = 0.f;
#pragma unroll 4
        for (int k = 0; k < splits; ++k) s += parts[k * all + i];
        const int64_t m = i / end.cols, n = i - m * end.cols;
        if (end.sums) {
            float *const sum = end.sums + m * end.lds + n;
            if (!end.first) s += *sum;
            if (!end.last) {
                *sum = s;
                continue;
            }
        }
        end.out[m * end.ld + n] = (T)(s * f);
    }
}

// Eight elements in 16 bits, or in pieces of which each takes what the ones before have left.
template <typename H, typename T, int PLANES>
__device__ __forceinline__ void pieces_of(const T (&v)[8], half8 (&o)[PLANES])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float x = (float)v[e];
#pragma unroll
        for (int k = 0; k < PLANES; ++k) {
            const H h = (H)x;
            o[k][e] = __builtin_bit_cast(uint16_t, h);
            x -= (float)h;
        }
    }
}

// Rows to whole lines of 64 elements (three bf16 pieces where PLANES is 3), zeros beyond the row and in rows that are not looked at:
// those whose label lies outside [0, V), and those from N on.
struct PackJob {
    const void *X;
    int64_t ldx, N, rows;
    int D, Dp;
    const int32_t *labels;  // NULL: all rows are looked at
    int64_t V;
    uint16_t *out;
    uint32_t groups;
};
// One array, or two in one launch: the second one's workgroups behind the first's.
template <typename T, typename H, int PLANES>
__global__ __launch_bounds__(256) void pack_kernel(PackJob first, PackJob second, uint32_t *zero, uint32_t zeros)
{
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < zeros; i += gridDim.x * 256) zero[i] = 0;
    const bool other = blockIdx.x >= first.groups;
    const PackJob j = other ? second : first;
    const int pieces = j.Dp / 8;
    const int64_t all = j.rows * pieces;
    for (int64_t i = (int64_t)(blockIdx.x - (other ? first.groups : 0)) * 256 + threadIdx.x; i < all; i += (int64_t)j.groups * 256) {
        const int64_t n = i / pieces;
        const int d = (int)(i - n * pieces) * 8;
        bool live = n < j.N;
        if (live && j.labels) live = j.labels[n] >= 0 && j.labels[n] < j.V;
        T v[8];
        if (live) {
            load8((const T *)j.X + n * j.ldx, d, j.D, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (T)0.f;
        }
        half8 o[PLANES];
        pieces_of<H>(v, o);
#pragma unroll
        for (int k = 0; k < PLANES; ++k) *reinterpret_cast<half8 *>(j.out + k * j.rows * j.Dp + n * j.Dp + d) = o[k];
    }
}

// The terms of 64 rows, and the largest |dloss| where it is asked for.
// exp(z - lse) is off by half a step of lse, 2^-8 at most below XENT_FAR.  Beyond it the logarithm of the sum is lost in lse little
// by little (masks of the type's lowest value on all classes: every class would have probability 1), and the
// rows of a group that has such a one are gone through anew: the logits of all classes in the products' order, with the same roundings, and
// from them the largest one and the sum of exponentials below it.  W is read as it lies, in full for every 64 rows; where those are few, in
// shares of the classes, whose last workgroup to end joins them, in order.  Other groups end at once (30000 rows: 4.6 us, a launch).
// All classes masked: 8192 rows x 65536 classes x 2048 in bf16 take 23.5 ms instead of 5.5, 30000 x 1024 x 256 in fp16 285 us instead of 121.
constexpr float XENT_FAR = 131072.f;
constexpr int TERMS_ROWS = 64, TERMS_WAVES = 8;
template <typename T>
struct TermsArgs {
    Logits z;  // of all classes
    const float *lse, *dloss;
    const uint16_t *X;  // packed
    int64_t plane;
    int Dp, D;
    const T *W;
    int64_t ldw;
    RowTerms *terms;
    uint32_t *top;  // NULL: not asked for
    int groups, shares;
    int64_t each;      // classes of a share
    uint64_t *parts;   // [groups][shares][64], and how many of a group have ended
    uint32_t *tickets;
};
template <typename T, typename H, int PLANES>
__global__ __launch_bounds__(64 * TERMS_WAVES, 2) void terms_kernel(TermsArgs<T> a)
{
    constexpr int MT = TERMS_ROWS / 16, WAVES = TERMS_WAVES;
    __shared__ float2 part[WAVES][TERMS_ROWS];
    __shared__ uint32_t largest[WAVES];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int group = blockIdx.x % (uint32_t)a.groups, share = blockIdx.x / (uint32_t)a.groups;
    const int64_t n0 = (int64_t)group * TERMS_ROWS, n = n0 + threadIdx.x;
    auto terms_of = [&](int64_t at) __attribute__((always_inline)) {
        const int32_t label = at < a.z.N ? a.z.labels[at] : -1;
        const float l = label >= 0 && label < a.z.V ? a.lse[at] : -__builtin_inff();
        return l != -__builtin_inff() ? RowTerms{l, 1.f, a.dloss[at], label} : RowTerms{__builtin_inff(), 0.f, 0.f, -1};
    };
    // (every eighth workgroup takes its followers' largest along: exchanges on one word go one after the other)
    const bool tops = a.top && share == 0 && group % WAVES == 0;
    RowTerms own{};
    if (w == 0 || tops) own = terms_of(n);
    if (tops) {
        uint32_t m = mag_bits(own.weight);
        for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
        if (lane == 0) largest[w] = m;
    }
    const int far = w == 0 && fabsf(own.shift) >= XENT_FAR && fabsf(own.shift) < __builtin_inff();
    const int any = __syncthreads_or(far);
    if (tops && threadIdx.x == 0) {
        uint32_t m = largest[0];
        for (int k = 1; k < WAVES; ++k) m = max(m, largest[k]);
        if (m) atomicMax(a.top, m);
    }
    if (!any) {
        if (w == 0 && share == 0) a.terms[n] = own;
        return;
    }
    float2 sum[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sum[i] = float2{-__builtin_inff(), 0.f};
    const int64_t end = min((share + 1) * a.each, a.z.V);
    for (int64_t v0 = share * a.each + 16 * w; v0 < end; v0 += 16 * WAVES) {
        const T *const row = a.W + min(v0 + r, a.z.V - 1) * a.ldw;
        float4v acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = float4v{0, 0, 0, 0};
        auto step = [&](int k, const T (&v)[8]) __attribute__((always_inline)) {
            half8 b[PLANES], x[PLANES][MT];
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    x[p][i] = *reinterpret_cast<const half8 *>(a.X + p * a.plane + (n0 + 16 * i + r) * a.Dp + k);
            pieces_of<H>(v, b);
            // (the order of pieces_kernel)
            constexpr int PRODUCTS = PLANES == 3 ? 6 : 1, PA[6] = {2, 1, 0, 1, 0, 0}, PB[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
            for (int s = 0; s < PRODUCTS; ++s)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    acc[i] = PLANES == 3 ? mma<H>(b[PB[s] % PLANES], x[PA[s] % PLANES][i], acc[i]) : mma<H>(b[0], x[0][i], acc[i]);
        };
        int k = 8 * q;
#pragma unroll 4
        for (; k < (a.D & ~31); k += 32) {
            T v[8];
#pragma unroll
            for (int c = 0; c < 8 / PIECE<T>; ++c) {
                const PieceOf<T> piece = row_piece(row + k + c * PIECE<T>);
#pragma unroll
                for (int e = 0; e < PIECE<T>; ++e) v[c * PIECE<T> + e] = piece[e];
            }
            step(k, v);
        }
        if (a.D & 31) {
            T v[8];
            load8(row, k, a.D, v);
            step(k, v);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float top = sum[i].x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[i][e] = fmaf(a.z.scale, acc[i][e], a.z.bias_of(v0 + 4 * q + e));
                top = fmaxf(top, acc[i][e]);
            }
            const float shift = top > -__builtin_inff() ? top : 0.f;
            float t = sum[i].y * exp2_of(sum[i].x - shift);
#pragma unroll
            for (int e = 0; e < 4; ++e) t += exp2_of(acc[i][e] - shift);
            sum[i] = float2{top, t};
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int d = 16; d < 64; d *= 2)
            sum[i] = SumEnd::joined(sum[i], float2{__shfl_xor(sum[i].x, d, 64), __shfl_xor(sum[i].y, d, 64)});
        if (q == 0) part[w][16 * i + r] = sum[i];
    }
    __syncthreads();
    if (w) return;
    float2 p = part[0][lane];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) p = SumEnd::joined(p, part[k][lane]);
    if (a.shares > 1) {
        uint64_t *const parts = a.parts + (int64_t)group * a.shares * TERMS_ROWS + lane;
        __hip_atomic_store(&parts[share * TERMS_ROWS], __builtin_bit_cast(uint64_t, p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        uint32_t ended = 0;
        if (lane == 0) ended = __hip_atomic_fetch_add(&a.tickets[group], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        if (__builtin_amdgcn_readfirstlane(ended) != (uint32_t)a.shares - 1) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        p = float2{-__builtin_inff(), 0.f};
        for (int k = 0; k < a.shares; ++k)
            p = SumEnd::joined(p, __builtin_bit_cast(float2, __hip_atomic_load(&parts[k * TERMS_ROWS], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
    }
    if (far) {
        own.shift = p.x;
        own.sum = p.y;
        own.weight /= p.y;
    }
    a.terms[n] = own;
}

// ---- calls -----------------------------------------------------------------------------------

struct XentPlan {
    bool direct;      // W is read where it lies
    bool few;         // one pass over it for all rows
    int planes;
    int64_t rows;     // N rounded up to whole stages
    int Dp;           // D rounded up to whole stages
    int64_t width;    // classes of a piece
    int64_t tiles;    // parts of a row's sums, of a piece
    // how products are cut: logits (or d), the rows' gradients, the classes'
    struct Cut {
        int tile, splits;
    } logits, rows_grad, classes_grad;
    size_t X, W, parts, running, label_logit, d, sums, shares, dbias, terms, parts_far, top, total;
    int shares_far;   // of the classes, where logits are gone through anew for a group of rows
};

using Large = Shape<8, 4, 2, 4>;   // 256 x 256, eight waves
using Middle = Shape<4, 2, 2, 4>;  // 128 x 128, eight waves (four of 64 x 64: 2 to 4 % more)
using Small = Shape<2, 2, 2, 2>;   // 64 x 64
constexpr int XENT_TILE = 64;      // columns that a sum's part stands for at least

constexpr int FEW_GROUPS = 256;    // workgroups of few rows' logits: one a compute unit

// Sums of logits of up to 32 rows (16, where half of D fills the registers).
static bool few_rows(int64_t N, int D) { return N <= 16 ? D <= 4096 : N <= 32 && D <= 2048; }

static bool rows_direct(ftk_dtype dtype, const void *p, int64_t ld, int D)
{
    return dtype != FTK_F32 && (uintptr_t)p % 16 == 0 && ld % 8 == 0 && D % 8 == 0 && ld < XENT_MAX_LD;
}

// Elements of k of a stage: three pieces come together.
constexpr int stage_of(int planes) { return planes == 3 ? 32 : XENT_STAGE; }

// How a product of rows x cols over so many stages of k is cut: the shape of the tiles, and shares of the stages where there are few.
// In microseconds: a stage of a tile of 256, 128 or 64 takes 1.85, 0.65 or 0.5 with a compute unit for itself, 1.1 and 0.85 where
// two and four share one, and begin and end take some more; joining shares is a launch and moves them once.
static XentPlan::Cut cut_of(int planes, int64_t rows, int64_t cols, int64_t k, bool shares)
{
    static const struct {
        int planes, tile, at_once;
        double ends, alone, shared;
    } shapes[] = {{1, 256, 1, 7, 1.85, 1.85}, {1, 128, 2, 5, 0.65, 0.55}, {1, 64, 4, 4, 0.5, 0.21}, 
                  {3, 128, 1, 4.5, 1.1, 1.1}, {3, 64, 2, 4, 0.6, 0.43}};
    const int64_t stages = ceil_div(k, stage_of(planes));
    XentPlan::Cut best{64, 1};
    double least = 1e300;
    for (const auto &s : shapes) {
        if (s.planes != planes) continue;
        const int64_t tiles = ceil_div(rows, s.tile) * ceil_div(cols, s.tile);
        for (int splits = 1; splits <= (shares ? 64 : 1) && splits * 4 - 3 <= stages; ++splits) {
            if (splits > 1 && tiles * splits > 256 * s.at_once) break;
            const int64_t groups = ceil_div(tiles * splits, 256);  // of a compute unit
            const double each = groups < s.at_once ? groups : s.at_once, stage = s.shared * each > s.alone ? s.shared * each : s.alone;
            const double t = (double)ceil_div(groups, s.at_once) * (s.ends + (double)ceil_div(stages, splits) * stage) +
                             (splits > 1 ? 5 + (double)rows * cols * (splits * 8 + 4) / 4e6 : 0);
            if (t < least) {
                least = t;
                best = {s.tile, splits};
            }
        }
    }
    return best;
}

static XentPlan plan_xent(ftk_dtype dtype, int64_t N, int64_t V, int D, bool grad, bool direct)
{
    XentPlan p;
    p.direct = direct;
    p.few = !grad && direct && few_rows(N, D);
    p.planes = dtype == FTK_F32 ? 3 : 1;
    p.rows = ceil_div(N > 0 ? N : 1, XENT_STAGE) * XENT_STAGE;  // (without rows gradients are zeros)
    p.Dp = (int)(ceil_div(D, XENT_STAGE) * XENT_STAGE);
    // d, or the packed rows of W, of a piece: about 256 MB
    const int64_t rows = direct ? p.rows : grad && p.rows > p.Dp ? p.rows : p.Dp;
    int64_t width = (128ll << 20) / p.planes / rows / 256 * 256;
    width = width < 256 ? 256 : width;
    const int64_t whole = ceil_div(V, 256) * 256;
    if (!grad) {
        // a part of the sums stands for 64 classes at least; 64 MB of them
        const int64_t parts = (8ll << 20) / (N > 0 ? N : 1) * XENT_TILE / 256 * 256;
        if (direct || parts < width) width = parts < 256 ? 256 : parts;
    }
    p.width = width < whole ? width : whole;
    // (pieces of equal width)
    p.width = ceil_div(ceil_div(V, ceil_div(V, p.width)), 256) * 256;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t a = at;
        at += align_up(bytes, 256);
        return a;
    };
    const int64_t classes = p.width < V ? p.width : V;
    p.logits = cut_of(p.planes, grad ? p.rows : N, classes, p.Dp, false);
    p.rows_grad = cut_of(p.planes, p.rows, D, classes, true);
    p.classes_grad = cut_of(p.planes, classes, D, p.rows, true);
    if (p.few) {
        p.tiles = ceil_div(V, 16) < FEW_GROUPS ? ceil_div(V, 16) : FEW_GROUPS;
        p.parts = take((size_t)N * p.tiles * 8);
        p.label_logit = take((size_t)N * 4);
        p.total = at;
        return p;
    }
    p.X = take((size_t)p.planes * p.rows * p.Dp * 2);
    p.W = direct ? at : take((size_t)p.planes * p.width * p.Dp * 2);
    p.parts = p.running = p.label_logit = p.d = p.sums = p.shares = p.dbias = p.terms = p.parts_far = p.top = at;
    p.shares_far = 1;
    if (grad) {
        p.d = take((size_t)p.planes * p.rows * p.width * 2);
        p.sums = dtype == FTK_F32 ? at : take((size_t)N * D * 4);
        const size_t rs = p.rows_grad.splits > 1 ? (size_t)p.rows_grad.splits * N * D * 4 : 0;
        const size_t cs = p.classes_grad.splits > 1 ? (size_t)p.classes_grad.splits * classes * D * 4 : 0;
        p.shares = take(rs > cs ? rs : cs);
        p.dbias = take((size_t)ceil_div(p.rows, XENT_TILE) * p.width * 4);
        p.terms = take((size_t)p.rows * sizeof(RowTerms));
        // (two workgroups a compute unit, each wave four tiles of classes at least)
        const int64_t groups = p.rows / TERMS_ROWS, wanted = groups < 512 ? 512 / groups : 1, most = ceil_div(V, 64 * TERMS_WAVES);
        p.shares_far = (int)(wanted < most ? wanted : most);
        p.parts_far = take(p.shares_far > 1 ? (size_t)p.rows * p.shares_far * 8 : 0);
        p.top = take((size_t)(1 + groups) * 4);  // and the groups' tickets
    } else {
        p.tiles = ceil_div(classes, p.logits.tile);
        p.parts = take((size_t)N * p.tiles * 8);
        p.running = p.width < V ? take((size_t)N * 8) : at;
        p.label_logit = take((size_t)N * 4);
    }
    p.total = at;
    return p;
}

template <typename S, typename H, int PLANES, bool AT, bool BT, typename End>
static ftk_status launch_shape(Product g, const End &end, hipStream_t st)
{
    const int64_t mt = ceil_div(g.a.outer, S::TM), nt = ceil_div(g.b.outer, S::TN), work = mt * nt * g.splits;
    if (work > 0x7fffffffLL) {
        set_error("too many tiles: %lld x %lld", (long long)mt, (long long)nt);
        return FTK_EINVAL;
    }
    g.mt = (uint32_t)mt;
    g.nt = (uint32_t)nt;
    if constexpr (PLANES == 3) {
        FTK_TRY(allow_lds<S::LDS3>((const void *)pieces_kernel<S, AT, BT, End>));
        pieces_kernel<S, AT, BT, End><<<(unsigned)work, S::THREADS, S::LDS3, st>>>(g, end);
    } else {
        FTK_TRY(allow_lds<S::LDS>((const void *)product_kernel<S, H, AT, BT, End>));
        product_kernel<S, H, AT, BT, End><<<(unsigned)work, S::THREADS, S::LDS, st>>>(g, end);
    }
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

template <typename H, int PLANES, bool AT, bool BT, typename End>
static ftk_status launch_product(const Product &g, int tile, const End &end, hipStream_t st)
{
    if constexpr (PLANES == 1)
        if (tile == 256) return launch_shape<Large, H, PLANES, AT, BT>(g, end, st);
    if (tile == 128) return launch_shape<Middle, H, PLANES, AT, BT>(g, end, st);
    return launch_shape<Small, H, PLANES, AT, BT>(g, end, st);
}

// A gradient's product, in shares where it is cut into them; their joining takes the bias' gradient along.
template <typename H, int PLANES, bool AT, typename T>
static ftk_status launch_gradient(Product g, const XentPlan::Cut &cut, const StoreEnd<T> &end, float *shares, BiasJob &bias, hipStream_t st)
{
    g.splits = cut.splits;
    if (cut.splits == 1) return launch_product<H, PLANES, AT, true>(g, cut.tile, end, st);
    FTK_TRY((launch_product<H, PLANES, AT, true>(g, cut.tile, PartEnd{shares, end.rows, end.cols}, st)));
    const int64_t groups = ceil_div(end.rows * end.cols, 256);
    if (groups == 0) return FTK_OK;
    const uint32_t join = groups < 2048 ? groups : 2048;
    join_kernel<T><<<join + (unsigned)ceil_div(bias.n, 16), 256, 0, st>>>(shares, cut.splits, end, join, bias);
    FTK_TRY_HIP(hipGetLastError());
    bias.n = 0;
    return FTK_OK;
}

template <typename T, typename H, int PLANES>
static ftk_status launch_pack(PackJob first, PackJob second, uint32_t *zero, uint32_t zeros, hipStream_t st)
{
    for (PackJob *j : {&first, &second}) {
        const int64_t groups = ceil_div(j->rows * (j->Dp / 8), 256);
        j->groups = (uint32_t)(groups < 4096 ? groups : 4096);
    }
    if (first.groups + second.groups == 0) return FTK_OK;
    pack_kernel<T, H, PLANES><<<first.groups + second.groups, 256, 0, st>>>(first, second, zero, zeros);
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

struct XentCall {
    const void *X, *W;
    int64_t ldx, N, ldw, V;
    int D;
    const float *bias;
    float scale;
    const int32_t *labels;
    uint8_t *ws;
    XentPlan p;
    hipStream_t st;
    PackJob rows_job() const { return PackJob{X, ldx, N, p.rows, D, p.Dp, labels, V, (uint16_t *)(ws + p.X), 0}; }
    // One piece's rows of W: packed, in one launch with `rows` (the first piece: those of X), or where they lie.
    template <typename T, typename H, int PLANES>
    ftk_status classes(int64_t first, int64_t n, const PackJob &rows, uint32_t *zero, uint32_t zeros, Operand &along, Operand &across) const
    {
        PackJob job{};
        if (p.direct) {
            const uint16_t *w = (const uint16_t *)W + first * ldw;
            along = Operand{w, ldw, 0, n, D};
            across = Operand{w, ldw, 0, D, n};
        } else {
            uint16_t *w = (uint16_t *)(ws + p.W);
            const int64_t rows = ceil_div(n, XENT_STAGE) * XENT_STAGE;
            job = PackJob{(const T *)W + first * ldw, ldw, n, rows, D, p.Dp, nullptr, 0, w, 0};
            along = Operand{w, p.Dp, rows * p.Dp, n, p.Dp};
            across = Operand{w, p.Dp, rows * p.Dp, p.Dp, rows};
        }
        return launch_pack<T, H, PLANES>(rows, job, zero, zeros, st);
    }
};

static ftk_status launch_loss(const XentCall &c, const SumEnd &end, float2 *running, bool first, bool last, float *loss, float *lse)
{
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        xent_loss_kernel<L><<<(unsigned)ceil_div(c.N, 256 / L), 256, 0, c.st>>>(end.parts, end.tiles, running, first, last, end.label_logit,
                                                                              c.labels, c.N, c.V, loss, lse);
        FTK_TRY_HIP(hipGetLastError());
        return FTK_OK;
    };
    // (two parts a lane where there are few)
    if (end.tiles <= 8) return go(std::integral_constant<int, 4>{});
    return end.tiles <= 64 ? go(std::integral_constant<int, 16>{}) : go(std::integral_constant<int, 64>{});
}

template <typename H, int MT, int RUN>
static ftk_status launch_few_shape(const XentCall &c, SumEnd end, float *loss, float *lse)
{
    const int64_t tiles = ceil_div(c.V, 16 * (16 / RUN / MT));
    end.tiles = tiles < FEW_GROUPS ? tiles : FEW_GROUPS;
    xent_few_kernel<H, MT, RUN><<<(unsigned)end.tiles, 512, 0, c.st>>>((const H *)c.X, c.ldx, (const H *)c.W, c.ldw, c.D, end);
    FTK_TRY_HIP(hipGetLastError());
    return launch_loss(c, end, nullptr, true, true, loss, lse);
}
template <typename H>
static ftk_status launch_few(const XentCall &c, const SumEnd &end, float *loss, float *lse)
{
    if (c.N > 16) return c.D <= 1024 ? launch_few_shape<H, 2, 4>(c, end, loss, lse) : launch_few_shape<H, 2, 8>(c, end, loss, lse);
    if (c.D <= 1024) return launch_few_shape<H, 1, 4>(c, end, loss, lse);
    return c.D <= 2048 ? launch_few_shape<H, 1, 8>(c, end, loss, lse) : launch_few_shape<H, 1, 16>(c, end, loss, lse);
}

template <typename T, typename H, int PLANES>
static ftk_status xent_forward(const XentCall &c, float *loss, float *lse)
{
    const XentPlan &p = c.p;
    float2 *parts = (float2 *)(c.ws + p.parts);
    float *label_logit = (float *)(c.ws + p.label_logit);
    if constexpr (PLANES == 1) {
        if (p.few) {
            const SumEnd end{Logits{c.bias, c.labels, c.N, 0, c.V, c.V, c.scale}, parts, 0, label_logit};
            return launch_few<H>(c, end, loss, lse);
        }
    }
    uint16_t *x = (uint16_t *)(c.ws + p.X);
    Product g;
    // (rows of whole stages are read where they lie: what an ignored one holds stays in its own sums, which are not looked at)
    const bool direct = PLANES == 1 && p.direct && c.D % XENT_STAGE == 0 && rows_direct(FTK_BF16, c.X, c.ldx, c.D);
    g.a = direct ? Operand{(const uint16_t *)c.X, c.ldx, 0, c.N, c.D} : Operand{x, p.Dp, p.rows * p.Dp, c.N, p.Dp};
    g.stages = p.Dp / stage_of(PLANES);
    g.splits = 1;
    const int tile = p.logits.tile;
    float2 *running = p.width < c.V ? (float2 *)(c.ws + p.running) : nullptr;
    for (int64_t first = 0; first < c.V; first += p.width) {
        const int64_t n = c.V - first < p.width ? c.V - first : p.width;
        Operand across;
        FTK_TRY((c.classes<T, H, PLANES>(first, n, first == 0 && !direct ? c.rows_job() : PackJob{}, nullptr, 0, g.b, across)));
        const SumEnd end{Logits{c.bias, c.labels, c.N, first, first + n, c.V, c.scale}, parts, ceil_div(n, tile), label_logit};
        FTK_TRY((launch_product<H, PLANES, false, false>(g, tile, end, c.st)));
        FTK_TRY(launch_loss(c, end, running, first == 0, first + n == c.V, loss, lse));
    }
    return FTK_OK;
}

template <typename T, typename H, int PLANES>
static ftk_status xent_backward(const XentCall &c, const float *lse, const float *dloss, T *dX, int64_t lddx, T *dW, int64_t lddw,
                                float *dbias)
{
    const XentPlan &p = c.p;
    uint16_t *x = (uint16_t *)(c.ws + p.X), *d = (uint16_t *)(c.ws + p.d);
    uint32_t *zeros = (uint32_t *)(c.ws + p.top), *top = std::is_same<T, _Float16>::value ? zeros : nullptr;
    const int groups = (int)(p.rows / TERMS_ROWS);
    float *parts = (float *)(c.ws + p.dbias), *shares = (float *)(c.ws + p.shares);
    RowTerms *terms = (RowTerms *)(c.ws + p.terms);
    constexpr int K = stage_of(PLANES);
    for (int64_t first = 0; first < c.V; first += p.width) {
        const int64_t n = c.V - first < p.width ? c.V - first : p.width, np = ceil_div(n, XENT_STAGE) * XENT_STAGE;
        const int64_t plane = p.rows * p.width;
        Operand along, across;
        FTK_TRY((c.classes<T, H, PLANES>(first, n, first == 0 ? c.rows_job() : PackJob{}, zeros, first == 0 ? 1 + groups : 0, along,
                                         across)));
        if (first == 0) {
            const int64_t each = ceil_div(ceil_div(c.V, p.shares_far), 16 * TERMS_WAVES) * (16 * TERMS_WAVES);
            const TermsArgs<T> args{Logits{c.bias, c.labels, c.N, 0, c.V, c.V, c.scale}, lse, dloss, x, p.rows * p.Dp, p.Dp, c.D, (const T *)c.W, c.ldw,
                                    terms, top, groups, p.shares_far, each, (uint64_t *)(c.ws + p.parts_far), zeros + 1};
            terms_kernel<T, H, PLANES><<<(unsigned)(groups * p.shares_far), 64 * TERMS_WAVES, 0, c.st>>>(args);
            FTK_TRY_HIP(hipGetLastError());
        }
        Product g{Operand{x, p.Dp, p.rows * p.Dp, p.rows, p.Dp}, along, 0, 0, p.Dp / K, 1};
        const int tile = p.logits.tile;
        const GradEnd<H, PLANES> grad{Logits{c.bias, c.labels, c.N, first, first + n, c.V, c.scale}, terms, top, d, p.width, plane, p.rows,
                                      dbias ? parts : nullptr};
        FTK_TRY((launch_product<H, PLANES, false, false>(g, tile, grad, c.st)));
        BiasJob bias{parts, p.width, (int)ceil_div(p.rows, tile), dbias ? n : 0, dbias ? dbias + first : nullptr};
        if (dX) {
            Product r{Operand{d, p.width, plane, p.rows, np}, across, 0, 0, (int)ceil_div(n, K), 1};
            const bool one = p.width >= c.V;
            // (in 32 bits dX itself holds them)
            float *sums = one ? nullptr : PLANES == 3 ? (float *)dX : (float *)(c.ws + p.sums);
            StoreEnd<T> end{dX, lddx, c.N, c.D, sums, PLANES == 3 ? lddx : c.D, first == 0, first + n == c.V, c.scale, top};
            FTK_TRY((launch_gradient<H, PLANES, false>(r, p.rows_grad, end, shares, bias, c.st)));
        }
        if (dW) {
            Product r{Operand{d, p.width, plane, np, p.rows}, Operand{x, p.Dp, p.rows * p.Dp, p.Dp, p.rows}, 0, 0,
                      (int)(p.rows / K), 1};
            StoreEnd<T> end{dW + first * lddw, lddw, n, c.D, nullptr, 0, true, true, c.scale, top};
            FTK_TRY((launch_gradient<H, PLANES, true>(r, p.classes_grad, end, shares, bias, c.st)));
        }
        if (bias.n) {
            dbias_kernel<<<(unsigned)ceil_div(bias.n, 16), 256, 0, c.st>>>(bias);
            FTK_TRY_HIP(hipGetLastError());
        }
    }
    return FTK_OK;
}

static ftk_status check_xent(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *W, int64_t ldw, int64_t V, int32_t D,
                             const float *bias, double scale, const int32_t *labels)
{
    FTK_TRY(check_mx_type(dtype));
    if (N < 0 || N > 0x7fffffffLL || V < 1 || V > 0x7fffffffLL || D < 1 || D > XENT_MAX_D) {
        set_error("need 0 <= N < 2^31, 1 <= V < 2^31, 1 <= D <= %d (got N=%lld V=%lld D=%d)", XENT_MAX_D, (long long)N, (long long)V, D);
        return FTK_EINVAL;
    }
    if (ldx < D || ldw < D) {
        set_error("row strides %lld of X and %lld of W must be at least D = %d", (long long)ldx, (long long)ldw, D);
        return FTK_EINVAL;
    }
    if (!isfinite(scale)) {
        set_error("scale must be finite (got %g)", scale);
        return FTK_EINVAL;
    }
    if (N > 0) {
        FTK_TRY(check_ptr(X, dtype_size(dtype), "X"));
        FTK_TRY(check_ptr(labels, 4, "labels"));
    }
    FTK_TRY(check_ptr(W, dtype_size(dtype), "W"));
    if (bias) FTK_TRY(check_ptr(bias, 4, "bias"));
    return FTK_OK;
}

}  // namespace ftk

using namespace ftk;

extern "C" {

int64_t ftk_xent_workspace_bytes(ftk_dtype dtype, int64_t N, int64_t V, int32_t D, int32_t grad)
{
    if (check_mx_type(dtype) != FTK_OK) return -1;
    if (N < 0 || N > 0x7fffffffLL || V < 1 || V > 0x7fffffffLL || D < 1 || D > XENT_MAX_D) {
        set_error("need 0 <= N < 2^31, 1 <= V < 2^31, 1 <= D <= %d (got N=%lld V=%lld D=%d)", XENT_MAX_D, (long long)N, (long long)V, D);
        return -1;
    }
    // for any address and stride of W
    const size_t packed = plan_xent(dtype, N, V, D, grad != 0, false).total, direct = plan_xent(dtype, N, V, D, grad != 0, true).total;
    return (int64_t)(packed > direct ? packed : direct);
}

ftk_status ftk_xent(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *W, int64_t ldw, int64_t V, int32_t D,
                    const float *bias, double scale, const int32_t *labels, float *loss, float *lse, void *workspace,
                    size_t workspace_bytes, void *hip_stream)
{
    FTK_TRY(check_xent(dtype, X, ldx, N, W, ldw, V, D, bias, scale, labels));
    if (N == 0) return FTK_OK;
    FTK_TRY(check_ptr(loss, 4, "loss"));
    FTK_TRY(check_ptr(lse, 4, "lse"));
    const XentPlan p = plan_xent(dtype, N, V, D, false, rows_direct(dtype, W, ldw, D));
    FTK_TRY(check_workspace(workspace, workspace_bytes, p.total));
    FTK_TRY(check_device());
    const XentCall c{X, W, ldx, N, ldw, V, D, bias, (float)scale, labels, (uint8_t *)workspace, p, (hipStream_t)hip_stream};
    switch (dtype) {
    case FTK_F32: return xent_forward<float, __bf16, 3>(c, loss, lse);
    case FTK_BF16: return xent_forward<__bf16, __bf16, 1>(c, loss, lse);
    default: return xent_forward<_Float16, _Float16, 1>(c, loss, lse);
    }
}

ftk_status ftk_xent_grad(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, const void *W, int64_t ldw, int64_t V, int32_t D,
                         const float *bias, double scale, const int32_t *labels, const float *lse, const float *dloss, void *dX,
                         int64_t lddx, void *dW, int64_t lddw, float *dbias, void *workspace, size_t workspace_bytes,
                         void *hip_stream)
{
    FTK_TRY(check_xent(dtype, X, ldx, N, W, ldw, V, D, bias, scale, labels));
    if (N > 0 && !dX && !dW && !dbias) {
        set_error("no gradient is asked for");
        return FTK_EINVAL;
    }
    if ((dX && lddx < D) || (dW && lddw < D)) {
        set_error("row strides %lld of dX and %lld of dW must be at least D = %d", (long long)lddx, (long long)lddw, D);
        return FTK_EINVAL;
    }
    if (N > 0) {
        FTK_TRY(check_ptr(lse, 4, "lse"));
        FTK_TRY(check_ptr(dloss, 4, "dloss"));
    }
    if (N == 0 && !dW && !dbias) return FTK_OK;  // (an empty dX may have no address)
    if (dX) FTK_TRY(check_ptr(dX, dtype_size(dtype), "dX"));
    if (dW) FTK_TRY(check_ptr(dW, dtype_size(dtype), "dW"));
    if (dbias) FTK_TRY(check_ptr(dbias, 4, "dbias"));
    const XentPlan p = plan_xent(dtype, N, V, D, true, rows_direct(dtype, W, ldw, D));
    FTK_TRY(check_workspace(workspace, workspace_bytes, p.total));
    FTK_TRY(check_device());
    const XentCall c{X, W, ldx, N, ldw, V, D, bias, (float)scale, labels, (uint8_t *)workspace, p, (hipStream_t)hip_stream};
    switch (dtype) {
    case FTK_F32: return xent_backward<float, __bf16, 3>(c, lse, dloss, (float *)dX, lddx, (float *)dW, lddw, dbias);
    case FTK_BF16: return xent_backward<__bf16, __bf16, 1>(c, lse, dloss, (__bf16 *)dX, lddx, (__bf16 *)dW, lddw, dbias);
    default: return xent_backward<_Float16, _Float16, 1>(c, lse, dloss, (_Float16 *)dX, lddx, (_Float16 *)dW, lddw, dbias);
    }
}

}  // extern "C"
