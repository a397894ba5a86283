// A gate over experts: probabilities of every row's logits, its k best experts, how evenly the rows use the experts, and the
// gradient of both.
//
//   p = softmax(z); labels: the k largest, ties to the lower index; weights: p there, or the softmax over them alone
//   T rows took part, counts[e] slots went to e, P_e = sum_t p_te / T, loss = E * sum_e counts[e] / (k T) * P_e
//   dz = p (c - <p, c>) with c_e = dloss E counts[e] / (k T^2), plus the weights' part: w_j (dw_j - <w, dw>) at the labels where
//   weights are normalised, p ([e = l_j] dw_j - <w, dw>) where not
//
// A row is read once, 16 bytes a lane and step, by 4, 16 or 64 lanes; what it needs stays in registers, so that memory is the
// bound where rows are many.  A lane keeps the same experts for all rows that pass, and so their sums of
// probabilities; those go through LDS and a table of one line a workgroup, in an order that the sizes alone set.
#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

constexpr int GATE_THREADS = 256, GATE_WAVES = GATE_THREADS / 64;
constexpr int GATE_MAX_EXPERTS = 8192, GATE_MAX_SLOTS = 64;
constexpr int GATE_MAX_GROUPS = 512;  // workgroups, lines of the table of sums
constexpr float NONE = -__builtin_inff();

struct GateArgs {
    const void *z;
    int64_t ldz, N;
    int E, k;
    bool normalise;
    int32_t *labels;
    float *weights, *lse;
    int32_t *counts;
    float *probs, *loss;
    // table of a line a workgroup: sums [E] and counts [E + 1]; NULL: one workgroup, which ends it all
    float *sums;
    int32_t *slots;
    int32_t *ticket;
};
struct GateGradArgs {
    const void *z;
    int64_t ldz, N;
    int E, k;
    bool normalise;
    const int32_t *labels;
    const float *weights, *lse;
    const int32_t *counts;
    const float *dweights, *dloss;  // NULL: none
    void *dz;
    int64_t ldd;
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// Largest over the L lanes of a group.
template <int L>
__device__ __forceinline__ float group_max(float v)
{
    v = fmaxf(v, dpp_move<0xB1>(v));
    if constexpr (L >= 4) v = fmaxf(v, dpp_move<0x4E>(v));
    if constexpr (L >= 8) v = fmaxf(v, dpp_move<0x141>(v));
    if constexpr (L >= 16) v = fmaxf(v, dpp_move<0x140>(v));
    if constexpr (L >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
    if constexpr (L >= 64) v = fmaxf(v, __shfl_xor(v, 32, 64));
    return v;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move_u(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v)
{
    v = max(v, dpp_move_u<0xB1>(v));
    if constexpr (L >= 4) v = max(v, dpp_move_u<0x4E>(v));
    if constexpr (L >= 8) v = max(v, dpp_move_u<0x141>(v));
    if constexpr (L >= 16) v = max(v, dpp_move_u<0x140>(v));
    if constexpr (L >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    if constexpr (L >= 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
    return v;
}

// Bits of a float in the floats' order, and back (the negative ones' are turned round).
__device__ __forceinline__ uint32_t ordered(float v)
{
    const int32_t b = (int32_t)__float_as_uint(v);
    return (uint32_t)b ^ ((uint32_t)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o)
{
    return __uint_as_float(o ^ ((uint32_t)((int32_t)~o >> 31) | 0x80000000u));
}

// The elements of a row that a lane has: pieces l, l + L, ... of P elements each; -infinity beyond the row.
template <typename T, int L, int NP>
struct RowShare {
    static constexpr int P = PIECE<T>, V = NP * P;
    static __device__ __forceinline__ int expert(int l, int i) { return (i / P * L + l) * P + i % P; }
    // (the pieces as they lie in memory: they can be requested a row ahead)
    static __device__ __forceinline__ void read(const T *row, int l, int E, PieceOf<T> (&q)[NP])
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = (i * L + l) * P;
            if (at + P <= E) {
                q[i] = row_piece(row + at);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) q[i][e] = at + e < E ? row[at + e] : (T)NONE;
            }
        }
    }
};

// The k best of a row, one after the other: at the end lane j of the group has number j.
//   16-bit logits: value and place fit one word.  A 32-bit number that comes from 16 bits has no more than 19 that
//   count; the other 13 hold the place, lower ones first.  32-bit logits: the largest value, then its lowest place.
template <typename T, int L, int NP>
__device__ __forceinline__ void best_of(const float (&v)[RowShare<T, L, NP>::V], int l, int k, float &value, int &label)
{
    using R = RowShare<T, L, NP>;
    value = NONE;
    label = -1;
    if constexpr (sizeof(T) == 2) {
        uint32_t last = 0xffffffffu;
        for (int j = 0; j < k; ++j) {
            uint32_t b = 0;
#pragma unroll
            for (int i = 0; i < R::V; ++i) {
                const uint32_t key = (ordered(v[i]) & 0xffffe000u) | (uint32_t)(GATE_MAX_EXPERTS - 1 - R::expert(l, i));
                b = max(b, key < last ? key : 0u);
            }
            last = group_max<L>(b);
            if (l == j) {
                const uint32_t o = last & 0xffffe000u;
                value = from_ordered((int32_t)o < 0 ? o : o | 0x1fffu);
                label = GATE_MAX_EXPERTS - 1 - (int)(last & 0x1fffu);
            }
        }
    } else {
        float lv = __builtin_inff();
        int le = -1;
        for (int j = 0; j < k; ++j) {
            float b = NONE;
#pragma unroll
            for (int i = 0; i < R::V; ++i) {
                const bool open = v[i] < lv || (v[i] == lv && R::expert(l, i) > le);
                b = fmaxf(b, open ? v[i] : NONE);
            }
            b = group_max<L>(b);
            uint32_t at = 0;
#pragma unroll
            for (int i = R::V - 1; i >= 0; --i) {
                const int e = R::expert(l, i);
                const bool open = v[i] == b && (b < lv || e > le);
                if (open) at = (uint32_t)(GATE_MAX_EXPERTS - e);
            }
            at = group_max<L>(at);
            le = GATE_MAX_EXPERTS - (int)at;
            lv = b;
            if (l == j) {
                value = b;
                label = le;
            }
        }
    }
}

// T, the share of every expert and the loss from sums and counts: at[e] and n[e] give them.
template <typename S, typename C>
__device__ __forceinline__ double gate_end(const GateArgs &a, int e, S sum, C count, int rows)
{
    const double T = rows > 0 ? rows : 1;
    const double mean = (double)sum / T;
    a.probs[e] = (float)mean;
    a.counts[e] = count;
    return mean * count * ((double)a.E / ((double)a.k * T));
}

template <typename T, int L, int NP>
__global__ __launch_bounds__(GATE_THREADS, (NP * PIECE<T> > 64 ? 1 : 2)) void gate_kernel(GateArgs a)
{
    using R = RowShare<T, L, NP>;
    extern __shared__ __align__(16) uint8_t gate_lds[];
    int *const slots = reinterpret_cast<int *>(gate_lds);  // [E + 1]
    float *const sums = reinterpret_cast<float *>(slots + a.E + 1);  // [E]
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane & (L - 1);
    for (int e = threadIdx.x; e <= a.E; e += GATE_THREADS) slots[e] = 0;
    if (a.ticket && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    __syncthreads();
    float acc[R::V];
#pragma unroll
    for (int i = 0; i < R::V; ++i) acc[i] = 0.f;
    constexpr int TOKENS = GATE_WAVES * (64 / L);
    const int64_t step = (int64_t)gridDim.x * TOKENS;
    // (all groups of a wave stay together; those beyond the last row have an empty one)
    int64_t t = (int64_t)blockIdx.x * TOKENS + w * (64 / L) + lane / L;
    int64_t first = (int64_t)blockIdx.x * TOKENS + w * (64 / L);
    PieceOf<T> q[NP];
    R::read((const T *)a.z + min(t, a.N - 1) * a.ldz, l, t < a.N ? a.E : 0, q);
    int rows = 0;
    for (; first < a.N; first += step, t += step) {
        float v[R::V];
#pragma unroll
        for (int i = 0; i < R::V; ++i) v[i] = (float)q[i / R::P][i % R::P] + 0.f;  // (one zero)
        const bool here = t < a.N;
        if (first + step < a.N) {
            const int64_t next = t + step;
            R::read((const T *)a.z + min(next, a.N - 1) * a.ldz, l, next < a.N ? a.E : 0, q);
        }
        float value;
        int label;
        best_of<T, L, NP>(v, l, a.k, value, label);
        float top = NONE;
#pragma unroll
        for (int i = 0; i < R::V; ++i) top = fmaxf(top, v[i]);
        top = group_max<L>(top);
        const bool some = top > NONE;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            v[i] = exp_of(v[i] - (some ? top : 0.f));
            sum += v[i];
        }
        sum = group_sum<L>(sum);
        // a NaN among the logits, or +infinity, makes the sum NaN: no labels, and weights and loss tell
        const bool bad = sum != sum;
        const float inv = some || bad ? 1.f / sum : 0.f;
#pragma unroll
        for (int i = 0; i < R::V; ++i) acc[i] += here ? v[i] * inv : 0.f;
        const bool held = value > NONE && !bad && l < a.k;
        const float ev = held ? exp_of(value - top) : 0.f;
        const float chosen = group_sum<L>(ev);
        if (here && l < a.k) {
            const float wt = bad ? __builtin_nanf("") : !held ? 0.f : a.normalise ? ev / chosen : ev * inv;
            a.weights[t * a.k + l] = wt;
            a.labels[t * a.k + l] = held ? label : -1;
            if (held) atomicAdd(&slots[label], 1);
        }
        if (here && l == 0) {
            a.lse[t] = bad ? __builtin_nanf("") : some ? top + logf(sum) : NONE;
            rows += some || bad;
        }
    }
    if (rows) atomicAdd(&slots[a.E], rows);
    // the groups of a wave, then the waves, one after the other
#pragma unroll
    for (int i = 0; i < R::V; ++i) {
        if constexpr (L <= 4) {
            acc[i] += __shfl_xor(acc[i], 4, 64);
            acc[i] += __shfl_xor(acc[i], 8, 64);
        }
        if constexpr (L <= 16) {
            acc[i] += __shfl_xor(acc[i], 16, 64);
            acc[i] += __shfl_xor(acc[i], 32, 64);
        }
    }
    for (int turn = 0; turn < GATE_WAVES; ++turn) {
        if (w == turn && lane < L) {
#pragma unroll
            for (int i = 0; i < R::V; ++i) {
                const int e = R::expert(l, i);
                if (e < a.E) sums[e] = turn ? sums[e] + acc[i] : acc[i];
            }
        }
        __syncthreads();
    }
    if (a.sums) {
        float *const line = a.sums + (int64_t)blockIdx.x * a.E;
        int32_t *const counts = a.slots + (int64_t)blockIdx.x * (a.E + 1);
        for (int e = threadIdx.x; e < a.E; e += GATE_THREADS) line[e] = sums[e];
        for (int e = threadIdx.x; e <= a.E; e += GATE_THREADS) counts[e] = slots[e];
        return;
    }
    const int total = slots[a.E];
    double part = 0;
    for (int e = threadIdx.x; e < a.E; e += GATE_THREADS) part += gate_end(a, e, sums[e], slots[e], total);
    part = group_sum<64>(part);
    __syncthreads();
    double *const parts = reinterpret_cast<double *>(gate_lds);
    if (lane == 0) parts[w] = part;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < GATE_WAVES; ++i) part += parts[i];
        a.counts[a.E] = total;
        *a.loss = (float)part;
    }
}

// The lines of all workgroups together: 64 experts a workgroup, a sixteenth of the lines a wave.  The last workgroup to
// end adds the parts of the loss up, in order.
constexpr int GATE_END_WAVES = 16;
__global__ __launch_bounds__(64 * GATE_END_WAVES) void gate_end_kernel(GateArgs a, int lines, double *parts)
{
    __shared__ float sums[GATE_END_WAVES][64];
    __shared__ int counts[GATE_END_WAVES][64], rows[GATE_END_WAVES];
    __shared__ bool last;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    float s = 0.f;
    int c = 0, T = 0;
#pragma unroll 4
    for (int b = w; b < lines; b += GATE_END_WAVES)
        if (e < a.E) {
            s += a.sums[(int64_t)b * a.E + e];
            c += a.slots[(int64_t)b * (a.E + 1) + e];
        }
    for (int b = threadIdx.x; b < lines; b += 64 * GATE_END_WAVES) T += a.slots[(int64_t)b * (a.E + 1) + a.E];
    for (int d = 32; d; d >>= 1) T += __shfl_xor(T, d, 64);
    sums[w][lane] = s;
    counts[w][lane] = c;
    if (lane == 0) rows[w] = T;
    __syncthreads();
    if (w) return;
    double total = 0, part = 0;
    T = 0;
    c = 0;
    for (int i = 0; i < GATE_END_WAVES; ++i) {
        total += sums[i][lane];
        c += counts[i][lane];
        T += rows[i];
    }
    if (e < a.E) part = gate_end(a, e, total, c, T);
    part = group_sum<64>(part);
    if (lane == 0) {
        __hip_atomic_store(&parts[blockIdx.x], part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        if (last) {
            double loss = 0;
            for (int i = 0; i < (int)gridDim.x; ++i)
                loss += __hip_atomic_load(&parts[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            a.counts[a.E] = T;
            *a.loss = (float)loss;
        }
    }
}

template <typename T, int L, int NP>
__global__ __launch_bounds__(GATE_THREADS, (NP * PIECE<T> > 64 ? 1 : 2)) void gate_grad_kernel(GateGradArgs a)
{
    using R = RowShare<T, L, NP>;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = lane & (L - 1);
    // what the loss asks of every probability of an expert
    float c[R::V];
    const float rows = (float)max(1, a.counts[a.E]);
    const float each = a.dloss ? *a.dloss * (float)a.E / ((float)a.k * rows) / rows : 0.f;
#pragma unroll
    for (int i = 0; i < R::V; ++i) {
        const int e = R::expert(l, i);
        c[i] = a.dloss && e < a.E ? each * (float)a.counts[e] : 0.f;
    }
    constexpr int TOKENS = GATE_WAVES * (64 / L);
    const int64_t step = (int64_t)gridDim.x * TOKENS;
    int64_t t = (int64_t)blockIdx.x * TOKENS + w * (64 / L) + lane / L;
    int64_t first = (int64_t)blockIdx.x * TOKENS + w * (64 / L);
    for (; first < a.N; first += step, t += step) {
        const bool here = t < a.N;
        const int64_t row = min(t, a.N - 1);
        PieceOf<T> q[NP];
        R::read((const T *)a.z + row * a.ldz, l, a.E, q);
        const float lse = a.lse[row];
        int label = -1;
        float add = 0.f, wt = 0.f;
        if (a.dweights && l < a.k) {
            label = a.labels[row * a.k + l];
            if (label >= 0) {
                wt = a.weights[row * a.k + l];
                add = wt * a.dweights[row * a.k + l];
            }
        }
        const float inner = group_sum<L>(add);
        if (a.normalise) add -= wt * inner;
        float p[R::V], dot = 0.f;
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            p[i] = lse == NONE ? 0.f : exp_of((float)q[i / R::P][i % R::P] - lse);
            dot = fmaf(p[i], c[i], dot);
        }
        dot = group_sum<L>(dot) + (a.normalise ? 0.f : inner);
#pragma unroll
        for (int i = 0; i < R::V; ++i) p[i] *= c[i] - dot;
        if (a.dweights)
            for (int j = 0; j < a.k; ++j) {
                const int from = (lane & ~(L - 1)) + j;
                const int e = __shfl(label, from, 64);
                const float d = __shfl(add, from, 64);
#pragma unroll
                for (int i = 0; i < R::V; ++i) p[i] += R::expert(l, i) == e ? d : 0.f;
            }
        if (!here) continue;
        T *const out = (T *)a.dz + t * a.ldd;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = (i * L + l) * R::P;
            PieceOf<T> o;
#pragma unroll
            for (int e = 0; e < R::P; ++e) o[e] = (T)p[i * R::P + e];
            if (at + R::P <= a.E) {
                put_piece(out + at, o);
            } else {
#pragma unroll
                for (int e = 0; e < R::P; ++e)
                    if (at + e < a.E) out[at + e] = o[e];
            }
        }
    }
}

// Lanes and pieces of a row: as few lanes as hold it in two pieces each, or in as many as there must be; a lane for each slot.
template <typename T, typename F>
static ftk_status with_share(int E, int k, F &&f)
{
    const int np = (E + PIECE<T> - 1) / PIECE<T>;
    auto go = [&](auto lanes, auto pieces) { return f(lanes, pieces); };
#define FTK_SHARE(L, NP) go(std::integral_constant<int, L>{}, std::integral_constant<int, NP>{})
    if (k <= 4 && np <= 4) return FTK_SHARE(4, 1);
    if (k <= 4 && np <= 8) return FTK_SHARE(4, 2);
    if (k <= 16 && np <= 16) return FTK_SHARE(16, 1);
    if (k <= 16 && np <= 32) return FTK_SHARE(16, 2);
    if (np <= 64) return FTK_SHARE(64, 1);
    if (np <= 128) return FTK_SHARE(64, 2);
    if (np <= 256) return FTK_SHARE(64, 4);
    if (np <= 512) return FTK_SHARE(64, 8);
    if (np <= 1024) return FTK_SHARE(64, 16);
    if constexpr (sizeof(T) == 4) return FTK_SHARE(64, 32);
#undef FTK_SHARE
    return FTK_EINVAL;  // (not reached: E <= GATE_MAX_EXPERTS)
}

static ftk_status check_gate(ftk_dtype dtype, int64_t N, int32_t E, int32_t k)
{
    FTK_TRY(check_mx_type(dtype));
    if (N < 0 || E < 1 || E > GATE_MAX_EXPERTS || k < 1 || k > GATE_MAX_SLOTS || k > E || N * k > 0x7fffffffLL || N > 0x7fffffffLL) {
        set_error("need N >= 0, 1 <= E <= %d, 1 <= k <= %d, k <= E and N * k < 2^31 (got N=%lld k=%d E=%d)", GATE_MAX_EXPERTS,
                  GATE_MAX_SLOTS, (long long)N, k, E);
        return FTK_EINVAL;
    }
    return FTK_OK;
}
static ftk_status check_rows_of(const void *p, ftk_dtype dtype, int64_t ld, int64_t N, int32_t E, const char *name)
{
    if (N == 0) return FTK_OK;
    if (ld < E) {
        set_error("row stride %lld of %s is less than E = %d", (long long)ld, name, E);
        return FTK_EINVAL;
    }
    return check_ptr(p, dtype_size(dtype), name);
}

// The table of sums, and what ends it.
struct GateTable {
    size_t sums, slots, parts, ticket, total;
};
static GateTable gate_table(int64_t groups, int E)
{
    GateTable t;
    t.sums = 0;
    t.slots = align_up((size_t)groups * E * 4, 256);
    t.parts = t.slots + align_up((size_t)groups * (E + 1) * 4, 256);
    t.ticket = t.parts + align_up((size_t)ceil_div(E, 64) * 8, 256);
    t.total = t.ticket + 256;
    return t;
}
// Rows that one workgroup ends in one launch.
static bool one_group(int64_t N) { return N <= FTK_ROUTE_GATE_FEW; }

}  // namespace ftk

using namespace ftk;

extern "C" {

size_t ftk_route_gate_workspace_bytes(int64_t N, int32_t E)
{
    if (N < 0 || N > 0x7fffffffLL || E < 1 || E > GATE_MAX_EXPERTS) {
        set_error("need 0 <= N < 2^31, 1 <= E <= %d (got N=%lld E=%d)", GATE_MAX_EXPERTS, (long long)N, E);
        return 0;
    }
    return one_group(N) ? 256 : gate_table(ceil_div(N, GATE_WAVES) < GATE_MAX_GROUPS ? ceil_div(N, GATE_WAVES) : GATE_MAX_GROUPS, E).total;
}

ftk_status ftk_route_gate(ftk_dtype dtype, const void *logits, int64_t ldz, int64_t N, int32_t E, int32_t k, int32_t normalise,
                          int32_t *labels, float *weights, float *lse, int32_t *counts, float *probs, float *loss,
                          void *workspace, size_t workspace_bytes, void *hip_stream)
{
    FTK_TRY(check_gate(dtype, N, E, k));
    FTK_TRY(check_rows_of(logits, dtype, ldz, N, E, "logits"));
    if (N > 0) {
        FTK_TRY(check_ptr(labels, 4, "labels"));
        FTK_TRY(check_ptr(weights, 4, "weights"));
        FTK_TRY(check_ptr(lse, 4, "lse"));
    }
    FTK_TRY(check_ptr(counts, 4, "counts"));
    FTK_TRY(check_ptr(probs, 4, "probs"));
    FTK_TRY(check_ptr(loss, 4, "loss"));
    const bool one = one_group(N);
    if (!one) FTK_TRY(check_workspace(workspace, workspace_bytes, ftk_route_gate_workspace_bytes(N, E)));
    FTK_TRY(check_device());
    hipStream_t st = (hipStream_t)hip_stream;
    GateArgs a{logits, ldz, N, E, k, normalise != 0, labels, weights, lse, counts, probs, loss, nullptr, nullptr, nullptr};
    if (N == 0) a.ldz = 0;
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return with_share<T>(E, k, [&](auto lanes, auto pieces) {
            constexpr int L = decltype(lanes)::value, NP = decltype(pieces)::value;
            const size_t lds = align_up((size_t)(2 * E + 1) * 4 + 32, 16);
            int64_t groups = ceil_div(N, GATE_WAVES * (64 / L));
            groups = one ? 1 : groups < GATE_MAX_GROUPS ? groups : GATE_MAX_GROUPS;
            double *parts = nullptr;
            if (!one) {
                const GateTable t = gate_table(groups, E);
                a.sums = (float *)((uint8_t *)workspace + t.sums);
                a.slots = (int32_t *)((uint8_t *)workspace + t.slots);
                a.ticket = (int32_t *)((uint8_t *)workspace + t.ticket);
                parts = (double *)((uint8_t *)workspace + t.parts);
            }
            FTK_TRY(allow_lds<(2 * GATE_MAX_EXPERTS + 1) * 4 + 48>((const void *)gate_kernel<T, L, NP>));
            gate_kernel<T, L, NP><<<(unsigned)groups, GATE_THREADS, lds, st>>>(a);
            FTK_TRY_HIP(hipGetLastError());
            if (!one) {
                gate_end_kernel<<<(unsigned)ceil_div(E, 64), 64 * GATE_END_WAVES, 0, st>>>(a, (int)groups, parts);
                FTK_TRY_HIP(hipGetLastError());
            }
            return FTK_OK;
        });
    });
}

ftk_status ftk_route_gate_grad(ftk_dtype dtype, const void *logits, int64_t ldz, int64_t N, int32_t E, int32_t k,
                               int32_t normalise, const int32_t *labels, const float *weights, const float *lse,
                               const int32_t *counts, const float *dweights, const float *dloss, void *dlogits, int64_t ldd,
                               void *hip_stream)
{
    FTK_TRY(check_gate(dtype, N, E, k));
    FTK_TRY(check_rows_of(logits, dtype, ldz, N, E, "logits"));
    FTK_TRY(check_rows_of(dlogits, dtype, ldd, N, E, "dlogits"));
    if (!dweights && !dloss) {
        set_error("neither dweights nor dloss is given");
        return FTK_EINVAL;
    }
    if (N == 0) return FTK_OK;
    FTK_TRY(check_ptr(lse, 4, "lse"));
    FTK_TRY(check_ptr(counts, 4, "counts"));
    if (dweights) {
        FTK_TRY(check_ptr(dweights, 4, "dweights"));
        FTK_TRY(check_ptr(labels, 4, "labels"));
        FTK_TRY(check_ptr(weights, 4, "weights"));
    }
    if (dloss) FTK_TRY(check_ptr(dloss, 4, "dloss"));
    FTK_TRY(check_device());
    const GateGradArgs a{logits, ldz, N, E, k, normalise != 0, labels, weights, lse, counts, dweights, dloss, dlogits, ldd};
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return with_share<T>(E, k, [&](auto lanes, auto pieces) {
            constexpr int L = decltype(lanes)::value, NP = decltype(pieces)::value;
            const int64_t groups = ceil_div(N, GATE_WAVES * (64 / L));
            gate_grad_kernel<T, L, NP><<<(unsigned)(groups < 2048 ? groups : 2048), GATE_THREADS, 0, (hipStream_t)hip_stream>>>(a);
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
    });
}

}  // extern "C"
