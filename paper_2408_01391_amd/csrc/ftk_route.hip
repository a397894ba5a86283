// Rows sorted by label and back: the plan (a stable counting sort of the slots by expert), the copy of the rows
// to their sorted places, the weighted sums that bring results back, and the gradients of both.
//
// All of it moves bytes: a plan reads 4 bytes a slot twice and writes 8, a copy reads every token's row once
// and writes it k times.  The copies therefore go by token, not by sorted row.
#include "ftk_quads.h"
#include "ftk_rows.h"

namespace ftk {

constexpr int ROUTE_THREADS = 256, ROUTE_WAVES = ROUTE_THREADS / 64;
constexpr int ROUTE_MAX_EXPERTS = 8192;  // one counter per wave and expert: 128 KB of a compute unit's 160
constexpr int ROUTE_CHUNK = FTK_ROUTE_FEW;  // slots of a workgroup, at least
constexpr int ROUTE_MAX_CHUNKS = 256;

struct RoutePlan {
    int S;       // slots
    int chunk;   // of a workgroup, a multiple of ROUTE_THREADS
    int chunks;  // workgroups
};
static RoutePlan plan_route(int64_t slots)
{
    RoutePlan p;
    p.S = (int)slots;
    p.chunk = ROUTE_CHUNK;
    if (ceil_div(slots, p.chunk) > ROUTE_MAX_CHUNKS)
        p.chunk = (int)(ceil_div(ceil_div(slots, ROUTE_MAX_CHUNKS), ROUTE_THREADS) * ROUTE_THREADS);
    p.chunks = (int)ceil_div(slots, p.chunk);
    return p;
}

// Slots of every expert among the slots of a workgroup.
__global__ __launch_bounds__(ROUTE_THREADS) void route_count_kernel(const int32_t *__restrict__ labels, int S, int chunk,
                                                                    int E, int32_t *__restrict__ table)
{
    extern __shared__ int cnt[];
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) cnt[e] = 0;
    __syncthreads();
    const int64_t s0 = (int64_t)blockIdx.x * chunk;
    const int n = (int)((int64_t)S - s0 < chunk ? (int64_t)S - s0 : chunk);
    for (int i = threadIdx.x; i < n; i += ROUTE_THREADS) {
        const uint32_t l = (uint32_t)labels[s0 + i];
        if (l < (uint32_t)E) atomicAdd(&cnt[l], 1);
    }
    __syncthreads();
    int32_t *row = table + (int64_t)blockIdx.x * E;
    for (int e = threadIdx.x; e < E; e += ROUTE_THREADS) row[e] = cnt[e];
}

// table[b][e] becomes the slots of e before workgroup b; totals[e] all of them.  A workgroup has 64 experts, a wave a
// sixteenth of the rows, all requested at once.
constexpr int PREFIX_WAVES = 16, PREFIX_ROWS = ROUTE_MAX_CHUNKS / PREFIX_WAVES;
__global__ __launch_bounds__(64 * PREFIX_WAVES) void route_prefix_kernel(int32_t *__restrict__ table, int chunks, int E,
                                                                         int32_t *__restrict__ totals)
{
    __shared__ int part[PREFIX_WAVES][64];
    const int lane = threadIdx.x & 63, e = blockIdx.x * 64 + lane, w = threadIdx.x >> 6;
    const int each = (chunks + PREFIX_WAVES - 1) / PREFIX_WAVES, b0 = w * each;  // each <= PREFIX_ROWS
    int v[PREFIX_ROWS], sum = 0;
#pragma unroll
    for (int i = 0; i < PREFIX_ROWS; ++i) v[i] = i < each && b0 + i < chunks && e < E ? table[(int64_t)(b0 + i) * E + e] : 0;
#pragma unroll
    for (int i = 0; i < PREFIX_ROWS; ++i) sum += v[i];
    part[w][lane] = sum;
    __syncthreads();
    if (e >= E) return;
    int run = 0;
    for (int i = 0; i < w; ++i) run += part[i][lane];
#pragma unroll
    for (int i = 0; i < PREFIX_ROWS; ++i) {
        if (i < each && b0 + i < chunks) table[(int64_t)(b0 + i) * E + e] = run;
        run += v[i];
    }
    if (w == PREFIX_WAVES - 1) totals[e] = run;
}

__device__ __forceinline__ int round_up(int v, int a) { return (v + a - 1) / a * a; }

// Exclusive prefix over the threads of a workgroup.
template <int WAVES>
__device__ __forceinline__ int block_prefix(int v, int *sums /* [WAVES], LDS */)
{
    const int lane = threadIdx.x & 63;
    int run = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(run, d, 64);
        if (lane >= d) run += o;
    }
    if (lane == 63) sums[threadIdx.x >> 6] = run;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        if (w < (int)(threadIdx.x >> 6)) before += sums[w];
    __syncthreads();
    return before + run - v;
}

// Place of a lane's slot, -1 without an expert.  The lanes of one label find each other by ballots over the label's bits, so
// a slot's rank is the count of lower lanes in its set, and the order of the slots is kept whatever the
// schedule; the first lane of a set moves its counter for all of them.  All lanes of a wave come here.
__device__ __forceinline__ int place_of(uint32_t l, int E, int ebits, int *counters)
{
    const int lane = threadIdx.x & 63;
    const bool routed = l < (uint32_t)E;
    unsigned long long same = __ballot(routed);
    for (int k = 0; k < ebits; ++k) {
        const unsigned long long m = __ballot((l >> k) & 1);
        same &= ((l >> k) & 1) ? m : ~m;
    }
    if (!routed) return -1;
    const int rank = __popcll(same & ((1ull << lane) - 1));
    int base = 0;
    if (rank == 0) base = atomicAdd(&counters[l], (int)__popcll(same));
    return __shfl(base, __ffsll(same) - 1, 64) + rank;
}

// Place of every slot.  cnt holds a row of counters for every wave, which has a contiguous quarter of the workgroup's
// slots: first how many of each expert it has, then where its next one goes, 64 slots at a time.
struct PlaceArgs {
    const int32_t *labels;
    int S, chunk, E, align, ebits;
    int64_t rows;
    const int32_t *table, *totals;  // NULL: this workgroup has all slots
    int32_t *offsets, *counts, *order, *pos;
};
__device__ __forceinline__ void place_slots(const PlaceArgs &a, int b, int blocks, bool write, int *cnt, int *sums,
                                            int *lds_pos /* or NULL */)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, E = a.E;
    const int64_t s0 = (int64_t)b * a.chunk;
    const int n = (int)((int64_t)a.S - s0 < a.chunk ? (int64_t)a.S - s0 : a.chunk);
    const int each = round_up((n + ROUTE_WAVES - 1) / ROUTE_WAVES, 64), i0 = w * each, i1 = min(n, i0 + each);
    // what has to be read is asked for at once: a lane's first labels, and the counts of a thread's first experts (a thread
    // has a run of consecutive ones)
    const int per = (E + ROUTE_THREADS - 1) / ROUTE_THREADS, e0 = min(E, tid * per), e1 = min(E, e0 + per);
    constexpr int KEEP = ROUTE_CHUNK / ROUTE_THREADS;
    uint32_t label[KEEP];
    int total[KEEP], before[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int i = i0 + k * 64 + lane;
        label[k] = i < i1 ? (uint32_t)a.labels[s0 + i] : 0xffffffffu;
        total[k] = a.totals && e0 + k < e1 ? a.totals[e0 + k] : 0;
        before[k] = a.table && e0 + k < e1 ? a.table[(int64_t)b * E + e0 + k] : 0;
    }
    for (int i = tid; i < ROUTE_WAVES * E; i += ROUTE_THREADS) cnt[i] = 0;
    __syncthreads();
    int *mine = cnt + w * E;
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (label[k] < (uint32_t)E) atomicAdd(&mine[label[k]], 1);
    for (int i = i0 + KEEP * 64 + lane; i < i1; i += 64) {
        const uint32_t l = (uint32_t)a.labels[s0 + i];
        if (l < (uint32_t)E) atomicAdd(&mine[l], 1);
    }
    __syncthreads();
    // f(expert of the run, its slots, those before this workgroup's)
    auto for_experts = [&](auto f) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (k < per) f(e0 + k, total[k], before[k]);
        for (int e = e0 + KEEP; e < e0 + per; ++e)
            f(e, a.totals && e < e1 ? a.totals[e] : 0, a.table && e < e1 ? a.table[(int64_t)b * E + e] : 0);
    };
    int need = 0;
    for_experts([&](int e, int t, int) {
        if (e >= e1) return;
        if (!a.totals)
            for (int v = 0; v < ROUTE_WAVES; ++v) t += cnt[v * E + e];
        need += round_up(t, a.align);
    });
    int off = block_prefix<ROUTE_WAVES>(need, sums);
    for_experts([&](int e, int t, int run) {
        int fill = 0, end = 0;  // rows that hold nothing, a wave's experts' one after the other
        if (e < e1) {
            int mine_all = 0;
            run += off;
            for (int v = 0; v < ROUTE_WAVES; ++v) {
                const int c = cnt[v * E + e];
                cnt[v * E + e] = run;
                run += c;
                mine_all += c;
            }
            if (!a.totals) t = mine_all;
            end = off + round_up(t, a.align);
            if (write && b == 0) {
                a.offsets[e] = off;
                if (a.counts) a.counts[e] = t;
                if (e == E - 1) a.offsets[E] = end;
            }
            fill = write && e % blocks == b ? off + t : end;
            off = end;
        }
        for (unsigned long long m = __ballot(fill < end); m; m &= m - 1) {
            const int from = __shfl(fill, __ffsll(m) - 1, 64), to = __shfl(end, __ffsll(m) - 1, 64);
            for (int64_t p = (int64_t)from + lane; p < to; p += 64) a.order[p] = -1;
        }
    });
    if (e1 == E && e0 < E) sums[0] = off;  // all sorted rows
    __syncthreads();
    if (write)
        for (int64_t p = sums[0] + (int64_t)b * ROUTE_THREADS + tid; p < a.rows; p += (int64_t)blocks * ROUTE_THREADS)
            a.order[p] = -1;
    auto place = [&](int i, uint32_t l) {  // 64 slots from i on
        const int p = place_of(l, E, a.ebits, mine);
        if (i + lane < i1) {
            if (write) {
                a.pos[s0 + i + lane] = p;
                if (p >= 0) a.order[p] = (int)(s0 + i + lane);
            }
            if (lds_pos) lds_pos[i + lane] = p;
        }
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (i0 + k * 64 < i1) place(i0 + k * 64, label[k]);
    for (int i = i0 + KEEP * 64; i < i1; i += 64) place(i, i + lane < i1 ? (uint32_t)a.labels[s0 + i + lane] : 0xffffffffu);
}

__global__ __launch_bounds__(ROUTE_THREADS) void route_place_kernel(PlaceArgs a)
{
    extern __shared__ int cnt[];
    __shared__ int sums[ROUTE_WAVES];
    place_slots(a, blockIdx.x, gridDim.x, true, cnt, sums, nullptr);
}

// ---- rows ------------------------------------------------------------------------------------

// A group of L lanes has a token (or, to fill, a sorted row); L covers the pieces of a row as far as 64 lanes go.
struct RowShape {
    int64_t N;
    int64_t rows;
    int k, D, np;  // np: pieces of a row
    bool stream;   // the result's rows are written past the caches
};

template <typename T, typename W>
__device__ __forceinline__ PieceOf<T> scale_piece(PieceOf<T> v, W w)
{
    using Acc = typename RowType<T>::Acc;
#pragma unroll
    for (int e = 0; e < PIECE<T>; ++e) v[e] = (T)((Acc)v[e] * (Acc)w);
    return v;
}

// zero rows [r0, rows) of out, those without a slot; a wave looks at 64 rows at a time
template <typename T>
__device__ __forceinline__ void fill_rows(const int32_t *order, const RowShape &h, int64_t wave, int64_t waves, T *out, int64_t ldo)
{
    const int lane = threadIdx.x & 63;
    const int64_t slots = h.N * h.k;
    for (int64_t r0 = wave * 64; r0 < h.rows; r0 += waves * 64) {
        bool empty = false;
        if (r0 + lane < h.rows) {
            const int32_t s = order[r0 + lane];
            empty = s < 0 || s >= slots;
        }
        unsigned long long m = __ballot(empty);
        while (m) {
            const int64_t r = r0 + __ffsll(m) - 1;
            m &= m - 1;
            T *o = out + r * ldo;
            if (h.D < PIECE<T>) {
                if (lane < h.D) o[lane] = (T)0.f;
            } else {
                for (int i = lane; i < h.np; i += 64) {
                    PieceOf<T> z = {};
                    put_piece(o + min(i * PIECE<T>, h.D - PIECE<T>), z, h.stream);
                }
            }
        }
    }
}

// A piece of a token's row to its k sorted places.
template <typename T, typename W>
__device__ __forceinline__ void copy_piece(const T *x, const int32_t *p, const W *w, int i, const RowShape &h, T *out, int64_t ldo)
{
    using Acc = typename RowType<T>::Acc;
    if (h.D < PIECE<T>) {
        const T v = x[i];
        for (int j = 0; j < h.k; ++j) {
            const int32_t r = p[j];
            if ((uint32_t)r < (uint64_t)h.rows) out[r * ldo + i] = w ? (T)((Acc)v * (Acc)w[j]) : v;
        }
    } else {
        const int c = min(i * PIECE<T>, h.D - PIECE<T>);
        const PieceOf<T> v = row_piece(x + c);
        for (int j = 0; j < h.k; ++j) {
            const int32_t r = p[j];
            if ((uint32_t)r < (uint64_t)h.rows) put_piece(out + r * ldo + c, w ? scale_piece<T>(v, w[j]) : v);
        }
    }
}

// Tokens' rows to their places; the last `fill` workgroups clear the rows without a slot.
template <typename T, typename W, int L>
__global__ __launch_bounds__(256) void route_gather_kernel(const T *__restrict__ X, int64_t ldx, RowShape h,
                                                           const int32_t *__restrict__ order,
                                                           const int32_t *__restrict__ pos,
                                                           const W *__restrict__ weights, T *__restrict__ out, int64_t ldo,
                                                           int fill)
{
    const int movers = gridDim.x - fill;
    if ((int)blockIdx.x >= movers) {
        fill_rows(order, h, (int64_t)(blockIdx.x - movers) * 4 + (threadIdx.x >> 6), (int64_t)fill * 4, out, ldo);
        return;
    }
    const int lane = threadIdx.x % L;
    const int64_t groups = (int64_t)movers * (256 / L);
    for (int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L; t < h.N; t += groups)
        for (int i = lane; i < h.np; i += L)
            copy_piece(X + t * ldx, pos + t * h.k, weights ? weights + t * h.k : nullptr, i, h, out, ldo);
}

// Few slots and no fill between experts: every workgroup works all places out by itself, which takes it less time than
// a second launch does, and copies its share of the rows.
template <typename T, int L>
__global__ __launch_bounds__(ROUTE_THREADS) void route_few_kernel(PlaceArgs a, const T *__restrict__ X, int64_t ldx, RowShape h,
                                                                  T *__restrict__ out, int64_t ldo)
{
    extern __shared__ int cnt[];
    __shared__ int sums[ROUTE_WAVES], places[FTK_ROUTE_FEW];
    place_slots(a, 0, 1, blockIdx.x == 0, cnt, sums, places);
    __syncthreads();
    const int lane = threadIdx.x % L, groups = gridDim.x * (256 / L), group = blockIdx.x * (256 / L) + threadIdx.x / L;
    for (int t = group; t < (int)h.N; t += groups)
        for (int i = lane; i < h.np; i += L)
            copy_piece(X + t * ldx, places + t * h.k, (const float *)nullptr, i, h, out, ldo);
    for (int64_t r = sums[0] + group; r < h.rows; r += groups)
        for (int i = lane; i < h.np; i += L) {
            T *o = out + r * ldo;
            if (h.D < PIECE<T>)
                o[i] = (T)0.f;
            else
                put_piece(o + min(i * PIECE<T>, h.D - PIECE<T>), PieceOf<T>{});
        }
}

// A token's sorted rows, times their weights, added up.  J slots at a time, whose loads are all under way before the
// first is used; a dropped slot reads row 0 and is left out by selection, so that nothing in it counts.
template <typename T, typename W, int L, int J>
__global__ __launch_bounds__(256) void route_combine_kernel(const T *__restrict__ Y, int64_t ldy, RowShape h,
                                                            const int32_t *__restrict__ pos, const W *__restrict__ weights,
                                                            T *__restrict__ out, int64_t ldo)
{
    using Acc = typename RowType<T>::Acc;
    const int lane = threadIdx.x % L;
    const int64_t groups = (int64_t)gridDim.x * (256 / L);
    for (int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L; t < h.N; t += groups) {
        for (int i = lane; i < h.np; i += L) {
            const bool whole = h.D >= PIECE<T>;
            const int c = whole ? min(i * PIECE<T>, h.D - PIECE<T>) : i;
            Acc acc[PIECE<T>];
#pragma unroll
            for (int e = 0; e < PIECE<T>; ++e) acc[e] = 0;
            for (int j0 = 0; j0 < h.k; j0 += J) {
                PieceOf<T> v[J];
                Acc w[J];
                bool in[J];
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int32_t r = j0 + j < h.k ? pos[t * h.k + j0 + j] : -1;
                    in[j] = (uint32_t)r < (uint64_t)h.rows;
                    w[j] = weights && in[j] ? (Acc)weights[t * h.k + j0 + j] : (Acc)1;
                    const T *y = Y + (in[j] ? r : 0) * ldy + c;
                    if (whole)
                        v[j] = row_piece(y);
                    else
                        v[j][0] = *y;
                }
#pragma unroll
                for (int j = 0; j < J; ++j) {
#pragma unroll
                    for (int e = 0; e < PIECE<T>; ++e) acc[e] = in[j] ? acc[e] + w[j] * (Acc)v[j][e] : acc[e];
                }
            }
            if (whole) {
                PieceOf<T> o;
#pragma unroll
                for (int e = 0; e < PIECE<T>; ++e) o[e] = (T)acc[e];
                put_piece(out + t * ldo + c, o, h.stream);
            } else {
                out[t * ldo + c] = (T)acc[0];
            }
        }
    }
}

// Both gradients of the weighted sum in one pass over dOut and Y.  The last piece of a ragged row shares
// elements with the one before: they are written twice and counted once.
template <typename T, typename W, int L, int J>
__global__ __launch_bounds__(256) void route_combine_grad_kernel(const T *__restrict__ G, int64_t ldg, const T *__restrict__ Y,
                                                                 int64_t ldy, RowShape h, const int32_t *__restrict__ order,
                                                                 const int32_t *__restrict__ pos,
                                                                 const W *__restrict__ weights, T *__restrict__ dY,
                                                                 int64_t ldd, W *__restrict__ dw, int fill)
{
    using Acc = typename RowType<T>::Acc;
    const int movers = gridDim.x - fill;
    if ((int)blockIdx.x >= movers) {
        fill_rows(order, h, (int64_t)(blockIdx.x - movers) * 4 + (threadIdx.x >> 6), (int64_t)fill * 4, dY, ldd);
        return;
    }
    const int lane = threadIdx.x % L;
    const int64_t groups = (int64_t)movers * (256 / L);
    for (int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L; t < h.N; t += groups) {
        for (int j0 = 0; j0 < h.k; j0 += J) {
            Acc dot[J], w[J];
            int32_t r[J];
            bool in[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                r[j] = j0 + j < h.k ? pos[t * h.k + j0 + j] : -1;
                in[j] = (uint32_t)r[j] < (uint64_t)h.rows;
                w[j] = in[j] ? (Acc)weights[t * h.k + j0 + j] : (Acc)0;
                dot[j] = 0;
            }
            for (int i = lane; i < h.np; i += L) {
                const bool whole = h.D >= PIECE<T>;
                const int c = whole ? min(i * PIECE<T>, h.D - PIECE<T>) : i;
                if (whole) {
                    const PieceOf<T> g = row_piece(G + t * ldg + c);
                    PieceOf<T> y[J];
#pragma unroll
                    for (int j = 0; j < J; ++j) y[j] = row_piece(Y + (in[j] ? r[j] : 0) * ldy + c);
                    const int twice = i * PIECE<T> - c;  // elements that the piece before has counted
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        if (!in[j]) continue;
#pragma unroll
                        for (int e = 0; e < PIECE<T>; ++e) dot[j] += e < twice ? (Acc)0 : (Acc)g[e] * (Acc)y[j][e];
                        put_piece(dY + r[j] * ldd + c, scale_piece<T>(g, w[j]), h.stream);
                    }
                } else {
                    const Acc g = (Acc)G[t * ldg + c];
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        if (!in[j]) continue;
                        dot[j] += g * (Acc)Y[r[j] * ldy + c];
                        dY[r[j] * ldd + c] = (T)(g * w[j]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const Acc s = group_sum<L>(dot[j]);
                if (lane == 0 && j0 + j < h.k) dw[t * h.k + j0 + j] = in[j] ? (W)s : (W)0;
            }
        }
    }
}

// Lanes of a row: as many as it has pieces, a power of two of 4 to 64.  (Fewer, where that leaves fewer of them idle in the last
// round, gain nothing: 333 floats, 84 pieces, weighted sum and its gradients 43 + 69 us with 64 lanes, 45 + 68
// with 32, 51 + 76 with 16, 83 + 118 with 4.)
static int row_lanes(int np)
{
    int l = 4;
    while (l < 64 && l < np) l <<= 1;
    return l;
}
template <typename F>
static ftk_status with_lanes(int np, F &&f)
{
    switch (row_lanes(np)) {
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    default: return f(std::integral_constant<int, 64>{});
    }
}
// slots of a token that are worked on together: all of them up to three, else four at a time
template <typename F>
static ftk_status with_slots(int k, F &&f)
{
    switch (k) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    default: return f(std::integral_constant<int, 4>{});
    }
}
static int row_grid(int64_t N, int lanes)
{
    const int64_t g = ceil_div(N, 256 / lanes);
    return (int)(g < 8192 ? g : 8192);
}
// workgroups that look for rows to clear: 256 rows each at a time
static int fill_grid(int64_t rows)
{
    const int64_t g = ceil_div(rows, 256);
    return (int)(g < 1024 ? g : 1024);
}

// ---- argument checks -------------------------------------------------------------------------

static ftk_status check_route(int64_t N, int32_t k, int32_t E, int32_t align)
{
    if (N < 0 || k < 1 || k > 64 || E < 1 || E > ROUTE_MAX_EXPERTS || align < 1 || align > 65536) {
        set_error("need N >= 0, 1 <= k <= 64, 1 <= E <= %d, 1 <= align <= 65536 (got N=%lld k=%d E=%d align=%d)",
                  ROUTE_MAX_EXPERTS, (long long)N, k, E, align);
        return FTK_EINVAL;
    }
    if (N > 0x7fffffffLL || N * k + (int64_t)E * (align - 1) > 0x7fffffffLL) {
        set_error("too many slots: N=%lld k=%d E=%d align=%d (need N * k + E * (align - 1) < 2^31)", (long long)N, k, E, align);
        return FTK_EINVAL;
    }
    return FTK_OK;
}
static int64_t route_rows(int64_t N, int k, int E, int align)
{
    const int64_t slots = N * k;
    return (slots + (slots < E ? slots : E) * (align - 1)) / align * align;
}

static ftk_status check_rows(ftk_dtype dtype, int64_t N, int32_t k, int32_t D, int64_t rows)
{
    if (!known_dtype(dtype)) {
        set_error("unknown dtype %d", (int)dtype);
        return FTK_EINVAL;
    }
    if (N < 0 || k < 1 || k > 64 || D < 1 || rows < 0) {
        set_error("need N >= 0, 1 <= k <= 64, D >= 1, rows >= 0 (got N=%lld k=%d D=%d rows=%lld)", (long long)N, k, D,
                  (long long)rows);
        return FTK_EINVAL;
    }
    if (D > (1 << 30) || rows > 0x7fffffffLL || N > 0x7fffffffLL || N * k > 0x7fffffffLL) {
        set_error("problem too large: N=%lld k=%d D=%d rows=%lld (need D <= 2^30, N * k and rows < 2^31)", (long long)N, k, D,
                  (long long)rows);
        return FTK_EINVAL;
    }
    return FTK_OK;
}
static ftk_status check_matrix(const void *p, size_t esz, int64_t ld, int32_t D, const char *name)
{
    FTK_TRY(check_ptr(p, esz, name));
    if (ld < D) {
        set_error("row stride %lld of %s is less than D = %d", (long long)ld, name, D);
        return FTK_EINVAL;
    }
    return FTK_OK;
}

static size_t route_workspace(int64_t slots, int E)
{
    const RoutePlan p = plan_route(slots);
    return p.chunks <= 1 ? 0 : align_up((size_t)(p.chunks + 1) * E * 4, 256);
}

static ftk_status check_plan(const int32_t *labels, int64_t N, int32_t k, int32_t E, int32_t align, int64_t rows,
                             int32_t *offsets, int32_t *counts, int32_t *order, int32_t *pos, void *ws, size_t ws_bytes)
{
    FTK_TRY(check_route(N, k, E, align));
    if (rows < route_rows(N, k, E, align) || rows > 0x7fffffffLL) {
        set_error("%lld sorted rows given, %lld may be needed", (long long)rows, (long long)route_rows(N, k, E, align));
        return FTK_EINVAL;
    }
    FTK_TRY(check_ptr(offsets, 4, "offsets"));
    if (counts) FTK_TRY(check_ptr(counts, 4, "counts"));
    if (N > 0) {
        FTK_TRY(check_ptr(labels, 4, "labels"));
        FTK_TRY(check_ptr(pos, 4, "pos"));
    }
    if (rows > 0) FTK_TRY(check_ptr(order, 4, "order"));
    const size_t need = route_workspace(N * k, E);
    if (need) FTK_TRY(check_workspace(ws, ws_bytes, need));
    return check_device();
}

static PlaceArgs place_args(const RoutePlan &p, const int32_t *labels, int E, int align, int64_t rows, int32_t *offsets,
                            int32_t *counts, int32_t *order, int32_t *pos)
{
    int ebits = 0;
    while ((1 << ebits) < E) ++ebits;
    return PlaceArgs{labels, p.S, p.chunk, E, align, ebits, rows, nullptr, nullptr, offsets, counts, order, pos};
}

static ftk_status launch_plan(const RoutePlan &p, PlaceArgs a, void *ws, hipStream_t st)
{
    const size_t lds = (size_t)ROUTE_WAVES * a.E * 4;
    if (lds > 65536) FTK_TRY(allow_lds<ROUTE_WAVES * ROUTE_MAX_EXPERTS * 4>((const void *)route_place_kernel));
    if (p.chunks > 1) {
        int32_t *totals = (int32_t *)ws, *table = totals + a.E;
        route_count_kernel<<<p.chunks, ROUTE_THREADS, (size_t)a.E * 4, st>>>(a.labels, p.S, p.chunk, a.E, table);
        route_prefix_kernel<<<(a.E + 63) / 64, 64 * PREFIX_WAVES, 0, st>>>(table, p.chunks, a.E, totals);
        a.table = table;
        a.totals = totals;
    }
    route_place_kernel<<<p.chunks > 1 ? p.chunks : 1, ROUTE_THREADS, lds, st>>>(a);
    FTK_TRY_HIP(hipGetLastError());
    return FTK_OK;
}

template <typename T>
using WeightOf = typename RowType<T>::Acc;

static ftk_status launch_gather(ftk_dtype dtype, const void *X, int64_t ldx, const RowShape &shape, const int32_t *order,
                                const int32_t *pos, const void *weights, void *out, int64_t ldo, hipStream_t st)
{
    return with_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        RowShape h = shape;
        h.np = row_pieces<T>(h.D);
        return with_lanes(h.np, [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            const int fill = fill_grid(h.rows);
            route_gather_kernel<T, WeightOf<T>, L><<<row_grid(h.N, L) + fill, 256, 0, st>>>(
                (const T *)X, ldx, h, order, pos, (const WeightOf<T> *)weights, (T *)out, ldo, fill);
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
    });
}

}  // namespace ftk

using namespace ftk;

extern "C" {

int64_t ftk_route_rows(int64_t N, int32_t k, int32_t E, int32_t align)
{
    if (check_route(N, k, E, align) != FTK_OK) return -1;
    return route_rows(N, k, E, align);
}

size_t ftk_route_workspace_bytes(int64_t N, int32_t k, int32_t E)
{
    if (check_route(N, k, E, 1) != FTK_OK) return 0;
    const size_t need = route_workspace(N * k, E);
    return need ? need : 256;
}

ftk_status ftk_route_plan(const int32_t *labels, int64_t N, int32_t k, int32_t E, int32_t align, int64_t rows,
                          int32_t *offsets, int32_t *counts, int32_t *order, int32_t *pos, void *workspace,
                          size_t workspace_bytes, void *hip_stream)
{
    FTK_TRY(check_plan(labels, N, k, E, align, rows, offsets, counts, order, pos, workspace, workspace_bytes));
    const RoutePlan p = plan_route(N * k);
    return launch_plan(p, place_args(p, labels, E, align, rows, offsets, counts, order, pos), workspace, (hipStream_t)hip_stream);
}

ftk_status ftk_route_gather(ftk_dtype dtype, const void *X, int64_t ldx, int64_t N, int32_t k, int32_t D,
                            const int32_t *order, const int32_t *pos, int64_t rows, const void *weights, void *out,
                            int64_t ldo, void *hip_stream)
{
    FTK_TRY(check_rows(dtype, N, k, D, rows));
    if (rows == 0) return FTK_OK;
    const size_t esz = dtype_size(dtype);
    FTK_TRY(check_matrix(out, esz, ldo, D, "out"));
    FTK_TRY(check_ptr(order, 4, "order"));
    if (N > 0) {
        FTK_TRY(check_matrix(X, esz, ldx, D, "X"));
        FTK_TRY(check_ptr(pos, 4, "pos"));
        if (weights) FTK_TRY(check_ptr(weights, esz == 8 ? 8 : 4, "weights"));
    }
    FTK_TRY(check_device());
    return launch_gather(dtype, X, ldx, RowShape{N, rows, k, D, 0, false}, order, pos, weights, out, ldo, (hipStream_t)hip_stream);
}

ftk_status ftk_route_dispatch(ftk_dtype dtype, const void *X, int64_t ldx, int32_t D, const int32_t *labels, int64_t N,
                              int32_t k, int32_t E, int32_t align, int64_t rows, int32_t *offsets, int32_t *counts,
                              int32_t *order, int32_t *pos, void *out, int64_t ldo, void *workspace,
                              size_t workspace_bytes, void *hip_stream)
{
    FTK_TRY(check_rows(dtype, N, k, D, rows));
    const size_t esz = dtype_size(dtype);
    if (rows > 0) FTK_TRY(check_matrix(out, esz, ldo, D, "out"));
    if (N > 0) FTK_TRY(check_matrix(X, esz, ldx, D, "X"));
    FTK_TRY(check_plan(labels, N, k, E, align, rows, offsets, counts, order, pos, workspace, workspace_bytes));
    hipStream_t st = (hipStream_t)hip_stream;
    const RoutePlan p = plan_route(N * k);
    const PlaceArgs a = place_args(p, labels, E, align, rows, offsets, counts, order, pos);
    const size_t lds = (size_t)ROUTE_WAVES * E * 4;
    if (rows > 0 && N * k <= FTK_ROUTE_FEW && align == 1 && lds <= 32768)
        return with_type(dtype, [&](auto tag) {
            using T = typename decltype(tag)::type;
            const RowShape h{N, rows, k, D, row_pieces<T>(D), false};
            return with_lanes(h.np, [&](auto lanes) {
                constexpr int L = decltype(lanes)::value;
                route_few_kernel<T, L><<<N > 0 ? row_grid(N, L) : 1, ROUTE_THREADS, lds, st>>>(a, (const T *)X, ldx, h, (T *)out, ldo);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            });
        });
    FTK_TRY(launch_plan(p, a, workspace, st));
    if (rows == 0) return FTK_OK;
    return launch_gather(dtype, X, ldx, RowShape{N, rows, k, D, 0, false}, order, pos, nullptr, out, ldo, st);
}

ftk_status ftk_route_combine(ftk_dtype dtype, const void *Y, int64_t ldy, int64_t rows, const int32_t *pos,
                             const void *weights, int64_t N, int32_t k, int32_t D, void *out, int64_t ldo,
                             void *hip_stream)
{
    FTK_TRY(check_rows(dtype, N, k, D, rows));
    if (N == 0) return FTK_OK;
    if (rows == 0) {
        set_error("no sorted rows for %lld tokens", (long long)N);
        return FTK_EINVAL;
    }
    const size_t esz = dtype_size(dtype);
    FTK_TRY(check_matrix(Y, esz, ldy, D, "Y"));
    FTK_TRY(check_matrix(out, esz, ldo, D, "out"));
    FTK_TRY(check_ptr(pos, 4, "pos"));
    if (weights) FTK_TRY(check_ptr(weights, esz == 8 ? 8 : 4, "weights"));
    FTK_TRY(check_device());
    hipStream_t st = (hipStream_t)hip_stream;
    return with_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        const RowShape h{N, rows, k, D, row_pieces<T>(D), streams_out((double)N * D * sizeof(T))};
        return with_lanes(h.np, [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            return with_slots(k, [&](auto slots) {
                constexpr int J = decltype(slots)::value;
                route_combine_kernel<T, WeightOf<T>, L, J><<<row_grid(N, L), 256, 0, st>>>(
                    (const T *)Y, ldy, h, pos, (const WeightOf<T> *)weights, (T *)out, ldo);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            });
        });
    });
}

ftk_status ftk_route_combine_grad(ftk_dtype dtype, const void *dOut, int64_t ldg, const void *Y, int64_t ldy,
                                  const int32_t *order, const int32_t *pos, int64_t rows, const void *weights,
                                  int64_t N, int32_t k, int32_t D, void *dY, int64_t ldd, void *dweights,
                                  void *hip_stream)
{
    FTK_TRY(check_rows(dtype, N, k, D, rows));
    if (rows == 0 && N > 0) {
        set_error("no sorted rows for %lld tokens", (long long)N);
        return FTK_EINVAL;
    }
    if (rows == 0) return FTK_OK;
    const size_t esz = dtype_size(dtype), wsz = esz == 8 ? 8 : 4;
    FTK_TRY(check_matrix(dY, esz, ldd, D, "dY"));
    FTK_TRY(check_ptr(order, 4, "order"));
    if (N > 0) {
        FTK_TRY(check_matrix(dOut, esz, ldg, D, "dOut"));
        FTK_TRY(check_matrix(Y, esz, ldy, D, "Y"));
        FTK_TRY(check_ptr(pos, 4, "pos"));
        FTK_TRY(check_ptr(weights, wsz, "weights"));
        FTK_TRY(check_ptr(dweights, wsz, "dweights"));
    }
    FTK_TRY(check_device());
    hipStream_t st = (hipStream_t)hip_stream;
    return with_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        const RowShape h{N, rows, k, D, row_pieces<T>(D), streams_out((double)rows * D * sizeof(T))};
        return with_lanes(h.np, [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            return with_slots(k, [&](auto slots) {
                constexpr int J = decltype(slots)::value;
                const int fill = fill_grid(rows);
                route_combine_grad_kernel<T, WeightOf<T>, L, J><<<row_grid(N, L) + fill, 256, 0, st>>>(
                    (const T *)dOut, ldg, (const T *)Y, ldy, h, order, pos, (const WeightOf<T> *)weights, (T *)dY, ldd,
                    (WeightOf<T> *)dweights, fill);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            });
        });
    });
}

}  // extern "C"
