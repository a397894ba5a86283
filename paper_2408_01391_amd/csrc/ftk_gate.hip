// A gate over experts: probabilities of every row's logits, its k best experts, how evenly the rows use the experts, and the
// gradient of both.
//
//   p = softmax(z); labels: the k largest, ties to the lower index; weights: p there, or the softmax over them alone
//   T rows took part, counts[e] slots went to e, P_e = sum_t p_te / T, loss = E * sum_e counts[e] / (k T) * P_e
//   dz = p (c - <p, c>) with c_e = dloss E counts[e] / (k T^2), plus the weights' part: w_j (dw_j - <w, dw>) at the labels where
//   weights are normalised, p ([e = l_j] dw_j - <w, dw>) where not
//
// A row is read once, 16 bytes a lane and step, by 4, 16, 64 or 256 lanes; what it needs stays in registers, so that memory is the
// bound where rows are many.  A lane keeps the same experts for all rows that pass, and so their sums of
// probabilities; those go through LDS and a table of one line a workgroup, in an order that the sizes alone set.
#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

constexpr int GATE_MAX_EXPERTS = 8192, GATE_MAX_SLOTS = 64;
constexpr int GATE_MAX_GROUPS = 512;  // workgroups, lines of the table of sums
constexpr int GATE_LIST = 8;  // experts that are found as a list
constexpr int GATE_PLACE = 4 * (GATE_LIST + 2);  // words that four waves exchange
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

constexpr float LOG2E = 1.44269504f;
// (of differences: a largest logit of the type's lowest value times LOG2E would be no number)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

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

// The lanes that share a row: 4, 16 or 64 of a wave, or a workgroup of four waves, which exchange through LDS; two turns
// alternate between two places there, so that each needs one barrier.
template <int L>
struct Group {
    static constexpr int WIDTH = L < 64 ? L : 64;
    uint32_t *place;  // [2][GATE_PLACE]
    int turn;
    template <typename V, typename F>
    __device__ __forceinline__ V joined(V v, F f)
    {
        if constexpr (L > 64) {
            V *const at = reinterpret_cast<V *>(place + (turn ^= 1) * GATE_PLACE);
            if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6 & 3] = v;
            __syncthreads();
            v = f(f(at[0], at[1]), f(at[2], at[3]));
        }
        return v;
    }
    __device__ __forceinline__ float sum(float v)
    {
        return joined(group_sum<WIDTH>(v), [](float x, float y) { return x + y; });
    }
    __device__ __forceinline__ float top(float v)
    {
        return joined(group_max<WIDTH>(v), [](float x, float y) { return fmaxf(x, y); });
    }
    __device__ __forceinline__ uint32_t top(uint32_t v)
    {
        return joined(group_max<WIDTH>(v), [](uint32_t x, uint32_t y) { return max(x, y); });
    }
};

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
        if (E == L * V) {
#pragma unroll
            for (int i = 0; i < NP; ++i) q[i] = row_piece(row + (i * L + l) * P);
            return;
        }
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

// The K largest keys so far in descending order, and one more.
template <int K>
__device__ __forceinline__ void insert_key(uint32_t (&m)[K], uint32_t x)
{
#pragma unroll
    for (int i = K - 1; i > 0; --i) m[i] = max(min(m[i - 1], m[i]), min(max(m[i - 1], m[i]), x));  // (the middle one)
    m[0] = max(m[0], x);
}
// The K largest of two such lists: what is larger of the first's number i and the second's K - 1 - i, put in order.
template <int K>
__device__ __forceinline__ void merge_keys(uint32_t (&m)[K], const uint32_t (&b)[K])
{
#pragma unroll
    for (int i = 0; i < K; ++i) m[i] = max(m[i], b[K - 1 - i]);
#pragma unroll
    for (int s = K / 2; s > 0; s /= 2)
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (!(i & s)) {
                const uint32_t hi = max(m[i], m[i + s]), lo = min(m[i], m[i + s]);
                m[i] = hi;
                m[i + s] = lo;
            }
}
template <int K, int CTRL>
__device__ __forceinline__ void merge_dpp(uint32_t (&m)[K])
{
    uint32_t b[K];
#pragma unroll
    for (int i = 0; i < K; ++i) b[i] = dpp_move_u<CTRL>(m[i]);
    merge_keys<K>(m, b);
}
template <int K>
__device__ __forceinline__ void merge_far(uint32_t (&m)[K], int d)
{
    uint32_t b[K];
#pragma unroll
    for (int i = 0; i < K; ++i) b[i] = (uint32_t)__shfl_xor((int)m[i], d, 64);
    merge_keys<K>(m, b);
}

// The softmax's largest logit and sum of exponentials below it from those of four waves.
__device__ __forceinline__ void join_softmax(const uint32_t *at, int stride, float &top, float &sum)
{
    float t[4], all = NONE;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = __uint_as_float(at[i * stride]);
        all = fmaxf(all, t[i]);
    }
    const float shift = all > NONE ? all : 0.f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += __uint_as_float(at[i * stride + 1]) * exp_of(t[i] - shift);
    top = all;
}

// The k best of a row: at the end lane j of the group has number j.
//   16-bit logits: value and place fit one word.  A 32-bit number that comes from 16 bits has no more than 19 that
//   count; the other 13 hold the place, lower ones first.  Up to eight are kept as lists, of a lane, then of pairs of lanes, and
//   so on; more are found one after the other, like the largest key below the last one.
//   32-bit logits: the largest value, then its lowest place, which is then closed.
// top, sum: the softmax's of the wave's part, and where a workgroup has the row (and K > 0), of the row.
// K: room of the list, 0 for none.  32-bit logits are overwritten.
template <typename T, int L, int NP, int K>
__device__ __forceinline__ void best_of(Group<L> &group, int l, int k, float (&v)[RowShare<T, L, NP>::V], float &top, float &sum, float &value, int &label)
{
    using R = RowShare<T, L, NP>;
    value = NONE;
    label = -1;
    if constexpr (sizeof(T) == 2) {
        auto key = [&](int i) __attribute__((always_inline)) {
            return (ordered(v[i]) & 0xffffe000u) | (uint32_t)(GATE_MAX_EXPERTS - 1 - R::expert(l, i));
        };
        uint32_t mine = 0;
        if constexpr (K > 0) {
            uint32_t m[K];
#pragma unroll
            for (int i = 0; i < K; ++i) m[i] = 0;
#pragma unroll
            for (int i = 0; i < R::V; ++i) insert_key<K>(m, key(i));
            merge_dpp<K, 0xB1>(m);
            if constexpr (L >= 4) merge_dpp<K, 0x4E>(m);
            if constexpr (L >= 8) merge_dpp<K, 0x141>(m);
            if constexpr (L >= 16) merge_dpp<K, 0x140>(m);
            if constexpr (L >= 32) merge_far<K>(m, 16);
            if constexpr (L >= 64) merge_far<K>(m, 32);
            if constexpr (L > 64) {
                // (with what the softmax needs of the other waves)
                uint32_t *const at = group.place + (group.turn ^= 1) * GATE_PLACE;
                const int w = threadIdx.x >> 6 & 3;
                if ((threadIdx.x & 63) == 0) {
                    at[w * (K + 2)] = __float_as_uint(top);
                    at[w * (K + 2) + 1] = __float_as_uint(sum);
#pragma unroll
                    for (int i = 0; i < K; ++i) at[w * (K + 2) + 2 + i] = m[i];
                }
                __syncthreads();
#pragma unroll
                for (int d = 1; d < 4; ++d) {
                    uint32_t b[K];
#pragma unroll
                    for (int i = 0; i < K; ++i) b[i] = at[((w + d) & 3) * (K + 2) + 2 + i];
                    merge_keys<K>(m, b);
                }
                join_softmax(at, K + 2, top, sum);
            }
#pragma unroll
            for (int j = 0; j < K; ++j) mine = l == j ? m[j] : mine;
        } else {
            uint32_t last = 0xffffffffu;
            for (int j = 0; j < k; ++j) {
                uint32_t b = 0;
#pragma unroll
                for (int i = 0; i < R::V; ++i) {
                    const uint32_t x = key(i);
                    b = max(b, x < last ? x : 0u);
                }
                last = group.top(b);
                mine = l == j ? last : mine;
            }
        }
        if (l < k) {
            const uint32_t o = mine & 0xffffe000u;
            value = from_ordered((int32_t)o < 0 ? o : o | 0x1fffu);
            label = GATE_MAX_EXPERTS - 1 - (int)(mine & 0x1fffu);
        }
    } else {
        for (int j = 0; j < k; ++j) {
            float b = NONE;
#pragma unroll
            for (int i = 0; i < R::V; ++i) b = fmaxf(b, v[i]);
            b = group.top(b);
            uint32_t at = 0;
#pragma unroll
            for (int i = R::V - 1; i >= 0; --i) at = v[i] == b ? (uint32_t)(GATE_MAX_EXPERTS - R::expert(0, i)) : at;
            at = group.top(at ? at - (uint32_t)(l * R::P) : 0u);
            const int e = GATE_MAX_EXPERTS - (int)at, mine = e - l * R::P;
#pragma unroll
            for (int i = 0; i < R::V; ++i) v[i] = R::expert(0, i) == mine ? NONE : v[i];
            if (l == j) {
                value = b;
                label = e;
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

// Waves of a workgroup: the more, the fewer lines the table has; rows that take many registers leave room for few.
template <typename T, int L, int NP>
constexpr int GATE_WAVES = L > 64 || NP * PIECE<T> > 16 ? 8 : 16;

// One pass: largest logit and sum of exponentials in registers, the k best beside them, the next row under way meanwhile.
// Reading the logits is the bound, with the exponentials and the lists close behind: 65536 rows of 256 in bf16, the eight best
// (34 MB read, 5 written): 22 us, 1.7 TB/s; 16384 rows of 4096 in fp16, the two best (134 MB): 47 us, 2.9 TB/s.  There eight pieces of a
// row (64 logits a lane) leave registers for two waves a SIMD, so that reading and arithmetic (27 us each) hardly overlap; a row by 256
// lanes of 16 logits, as in the gradient, was not tried.
template <typename T, int L, int NP, int K>
__global__ __launch_bounds__((64 * GATE_WAVES<T, L, NP>), (NP * PIECE<T> > 16 ? 2 : 4)) void gate_kernel(GateArgs a)
{
    using R = RowShare<T, L, NP>;
    constexpr int WAVES = GATE_WAVES<T, L, NP>, THREADS = 64 * WAVES, TOKENS = THREADS / L;
    extern __shared__ __align__(16) uint8_t gate_lds[];
    int *const slots = reinterpret_cast<int *>(gate_lds);  // [E + 1]
    float *const sums = reinterpret_cast<float *>(slots + a.E + 1);  // of every wave, or row at a time, [E]
    __shared__ uint32_t place[L > 64 ? TOKENS * 2 * GATE_PLACE : 1];
    Group<L> group{place + (L > 64 ? threadIdx.x / L * 2 * GATE_PLACE : 0), 0};
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l = threadIdx.x & (L - 1);
    for (int e = threadIdx.x; e <= a.E; e += THREADS) slots[e] = 0;
    if (a.ticket && blockIdx.x == 0 && threadIdx.x == 0) *a.ticket = 0;
    __syncthreads();
    float acc[R::V];
#pragma unroll
    for (int i = 0; i < R::V; ++i) acc[i] = 0.f;
    const int64_t step = (int64_t)gridDim.x * TOKENS;
    // (all groups of a wave, or of a workgroup, stay together; those beyond the last row have that one, and leave nothing)
    int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / L;
    int64_t first = (int64_t)blockIdx.x * TOKENS + (L > 64 ? 0 : w * (64 / Group<L>::WIDTH));
    PieceOf<T> q[NP];
    if (first < a.N) R::read((const T *)a.z + min(t, a.N - 1) * a.ldz, l, a.E, q);
    int rows = 0;
    for (; first < a.N; first += step, t += step) {
        float v[R::V];
#pragma unroll
        for (int i = 0; i < R::V; ++i) v[i] = (float)q[i / R::P][i % R::P] + 0.f;  // (one zero)
        const bool here = t < a.N;
        if (first + step < a.N) R::read((const T *)a.z + min(t + step, a.N - 1) * a.ldz, l, a.E, q);
        float value, top = NONE, sum = 0.f;
        int label;
        // (16-bit logits need not be kept beside their exponentials)
        constexpr bool LIST_FIRST = sizeof(T) == 2 && L <= 64;
        if constexpr (LIST_FIRST) best_of<T, L, NP, K>(group, l, a.k, v, top, sum, value, label);
#pragma unroll
        for (int i = 0; i < R::V; ++i) top = fmaxf(top, v[i]);
        // (where four waves have the row, each takes its own part's largest first)
        constexpr int W = Group<L>::WIDTH;
        top = group_max<W>(top);
        const bool any = top > NONE;
        const float own = any ? top : 0.f;
        float e[R::V];
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            e[i] = exp_of(v[i] - own);
            sum += e[i];
        }
        sum = group_sum<W>(sum);
        if constexpr (L > 64 && K == 0) {
            uint32_t *const at = group.place + (group.turn ^= 1) * GATE_PLACE;
            if (lane == 0) {
                at[2 * (w & 3)] = __float_as_uint(top);
                at[2 * (w & 3) + 1] = __float_as_uint(sum);
            }
            __syncthreads();
            join_softmax(at, 2, top, sum);
        }
        if constexpr (!LIST_FIRST) best_of<T, L, NP, K>(group, l, a.k, v, top, sum, value, label);
        const bool some = top > NONE;
        const float shift = some ? top : 0.f;
        // a NaN among the logits, or +infinity, makes the sum NaN: no labels, and weights and loss tell
        const bool bad = sum != sum;
        const float inv = some || bad ? 1.f / sum : 0.f;
        float mine = here ? inv : 0.f;
        if (L > 64) mine *= any || bad ? exp_of(own - shift) : 0.f;
#pragma unroll
        for (int i = 0; i < R::V; ++i) acc[i] = fmaf(e[i], mine, acc[i]);
        const bool held = value > NONE && !bad && l < a.k;
        const float ev = held ? exp_of(value - shift) : 0.f;
        const float chosen = group_sum<Group<L>::WIDTH>(ev);
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
    // the groups of a wave, then the waves in order
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
    if (L > 64 || lane < L) {
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            const int e = R::expert(l, i);
            if (e < a.E) sums[(L > 64 ? threadIdx.x / L : w) * a.E + e] = acc[i];
        }
    }
    __syncthreads();
    auto sum_of = [&](int e) __attribute__((always_inline)) {
        float s = sums[e];
#pragma unroll
        for (int i = 1; i < (L > 64 ? TOKENS : WAVES); ++i) s += sums[i * a.E + e];
        return s;
    };
    if (a.sums) {
        float *const line = a.sums + (int64_t)blockIdx.x * a.E;
        int32_t *const counts = a.slots + (int64_t)blockIdx.x * (a.E + 1);
        for (int e = threadIdx.x; e < a.E; e += THREADS) line[e] = sum_of(e);
        for (int e = threadIdx.x; e <= a.E; e += THREADS) counts[e] = slots[e];
        return;
    }
    const int total = slots[a.E];
    double part = 0;
    for (int e = threadIdx.x; e < a.E; e += THREADS) part += gate_end(a, e, sum_of(e), slots[e], total);
    part = group_sum<64>(part);
    __syncthreads();
    double *const parts = reinterpret_cast<double *>(gate_lds);
    if (lane == 0) parts[w] = part;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < WAVES; ++i) part += parts[i];
        a.counts[a.E] = total;
        *a.loss = (float)part;
    }
}

// The lines of all workgroups together: 32 experts a workgroup, a 32nd of the lines half a wave, sixteen of them under way at a
// time.  The last workgroup to end adds the parts of the loss up, in order.  A launch of its own, for the bandwidth of many
// workgroups: 256 lines of 4096 experts (8 MB) take 7.8 us.  The last workgroup of gate_kernel could add small tables up by itself, in the same
// order: 256 lines of 256 experts take 5.2 us here, of which a launch alone is 4.2.
constexpr int GATE_END_EXPERTS = 32, GATE_END_SHARES = 32, GATE_END_THREADS = GATE_END_EXPERTS * GATE_END_SHARES;
__global__ __launch_bounds__(GATE_END_THREADS) void gate_end_kernel(GateArgs a, int lines, double *parts)
{
    __shared__ float sums[GATE_END_SHARES][GATE_END_EXPERTS];
    __shared__ int counts[GATE_END_SHARES][GATE_END_EXPERTS], rows[GATE_END_THREADS / 64];
    const int lane = threadIdx.x & (GATE_END_EXPERTS - 1), share = threadIdx.x / GATE_END_EXPERTS, e = blockIdx.x * GATE_END_EXPERTS + lane;
    float s = 0.f;
    int c = 0, T = 0;
    for (int b = threadIdx.x; b < lines; b += GATE_END_THREADS) T += a.slots[(int64_t)b * (a.E + 1) + a.E];
    if (e < a.E) {
        for (int b0 = share; b0 < lines; b0 += 16 * GATE_END_SHARES) {
            float x[16];
            int y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int b = b0 + i * GATE_END_SHARES;
                x[i] = b < lines ? a.sums[(int64_t)b * a.E + e] : 0.f;
                y[i] = b < lines ? a.slots[(int64_t)b * (a.E + 1) + e] : 0;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s += x[i];
                c += y[i];
            }
        }
    }
    for (int d = 32; d; d >>= 1) T += __shfl_xor(T, d, 64);
    sums[share][lane] = s;
    counts[share][lane] = c;
    if ((threadIdx.x & 63) == 0) rows[threadIdx.x >> 6] = T;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    // (the first wave; its second half only fills it up)
    double total = 0, part = 0;
    T = 0;
    c = 0;
    for (int i = 0; i < GATE_END_SHARES; ++i) {
        total += sums[i][lane];
        c += counts[i][lane];
    }
    for (int i = 0; i < GATE_END_THREADS / 64; ++i) T += rows[i];
    if (e < a.E && threadIdx.x < GATE_END_EXPERTS) part = gate_end(a, e, total, c, T);
    part = group_sum<64>(part);
    int done = 0;
    if (threadIdx.x == 0) {
        __hip_atomic_store(&parts[blockIdx.x], part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        done = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (__builtin_amdgcn_readfirstlane(done) != (int)gridDim.x - 1) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    double loss = 0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 64) loss += __hip_atomic_load(&parts[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    loss = group_sum<64>(loss);
    if (threadIdx.x == 0) {
        a.counts[a.E] = T;
        *a.loss = (float)loss;
    }
}

// One pass again: probabilities from lse, which needs one sum over the row (<p, c>) rather than two, as 32-bit logits do.  Memory is the bound: 65536 rows of
// 256 in bf16 (67 MB and the labels' 8 MB): 20 us, 3.8 TB/s.
// What the labels add to a row's gradient goes through a row of LDS of the group's own, whose zeros are put back.
constexpr int GATE_GRAD_WAVES = 4;
template <typename T, int L, int NP>
__global__ __launch_bounds__(64 * GATE_GRAD_WAVES, (NP * PIECE<T> > 16 ? 2 : 4)) void gate_grad_kernel(GateGradArgs a)
{
    using R = RowShare<T, L, NP>;
    extern __shared__ __align__(16) uint8_t gate_lds[];
    __shared__ uint32_t place[L > 64 ? 2 * GATE_PLACE : 1];
    Group<L> group{place, 0};
    const int w = threadIdx.x >> 6, l = threadIdx.x & (L - 1);
    constexpr int TOKENS = 64 * GATE_GRAD_WAVES / L, WIDTH = L * R::V;
    float *const add_of = reinterpret_cast<float *>(gate_lds) + threadIdx.x / L * WIDTH;
#pragma unroll
    for (int i = 0; i < R::V; ++i) add_of[R::expert(l, i)] = 0.f;
    const int64_t step = (int64_t)gridDim.x * TOKENS;
    int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / L;
    int64_t first = L > 64 ? t : (int64_t)blockIdx.x * TOKENS + w * (64 / Group<L>::WIDTH);
    // a row's operands, which are requested a row ahead
    PieceOf<T> q[NP];
    float lse = 0.f, wt = 0.f, dw = 0.f;
    uint32_t label = ~0u;
    auto request = [&](int64_t row) __attribute__((always_inline)) {
        R::read((const T *)a.z + row * a.ldz, l, a.E, q);
        lse = a.lse[row];
        if (a.dweights && l < a.k) {
            label = (uint32_t)a.labels[row * a.k + l];
            wt = a.weights[row * a.k + l];
            dw = a.dweights[row * a.k + l];
        }
    };
    if (first < a.N) request(min(t, a.N - 1));
    // what the loss asks of every probability of an expert
    float c[R::V];
    const float rows = (float)max(1, a.counts[a.E]);
    const float each = a.dloss ? *a.dloss * (float)a.E / ((float)a.k * rows) / rows : 0.f;
#pragma unroll
    for (int i = 0; i < R::V; ++i) {
        const int e = R::expert(l, i);
        c[i] = a.dloss && e < a.E ? each * (float)a.counts[e] : 0.f;
    }
    for (; first < a.N; first += step, t += step) {
        const bool here = t < a.N, chosen = label < (uint32_t)a.E;
        const uint32_t at_label = label;
        const float shift = lse, w_here = wt;
        const bool none = lse == NONE;
        float p[R::V], add = chosen ? wt * dw : 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < R::V; ++i) p[i] = (float)q[i / R::P][i % R::P];
        if (first + step < a.N) request(min(t + step, a.N - 1));
        const float inner = group.sum(add);
        if (a.normalise) add = chosen ? add - w_here * inner : 0.f;
        if (chosen) atomicAdd(&add_of[at_label], add);
#pragma unroll
        for (int i = 0; i < R::V; ++i) {
            p[i] = exp_of(p[i] - shift);
            p[i] = none ? 0.f : p[i];
        }
        // where half a step of lse is no longer small: by their own sum (a row of masks of the type's lowest value).  16-bit gradients round
        // to 2^-11 of themselves at best, what lse is off by below 64 is 2^-19; in 32 bits it would be what bounds them
        constexpr float FAR = sizeof(T) == 2 ? 64.f : 1.f;
        if (__any(fabsf(shift) > FAR)) {
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < R::V; ++i) all += p[i];
            all = group.sum(all);
            all = none || !(fabsf(shift) > FAR) ? 1.f : 1.f / all;
#pragma unroll
            for (int i = 0; i < R::V; ++i) p[i] *= all;
        }
#pragma unroll
        for (int i = 0; i < R::V; ++i) dot = fmaf(p[i], c[i], dot);
        dot = group.sum(dot) + (a.normalise ? 0.f : inner);
        if (a.dweights) {
#pragma unroll
            for (int i = 0; i < R::V; ++i) p[i] = fmaf(p[i], c[i] - dot, add_of[R::expert(l, i)]);
            if constexpr (L > 64) __syncthreads();
            if (chosen) add_of[at_label] = 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < R::V; ++i) p[i] *= c[i] - dot;
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
template <typename T, bool GRAD, typename F>
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
    // (64 logits a lane leave the gradient no registers)
    if (np <= 512) return FTK_SHARE(GRAD ? 256 : 64, GRAD ? 2 : 8);
    if constexpr (sizeof(T) == 2) return FTK_SHARE(256, 4);
    else return FTK_SHARE(256, 8);
#undef FTK_SHARE
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
    t.ticket = t.parts + align_up((size_t)ceil_div(E, GATE_END_EXPERTS) * 8, 256);
    t.total = t.ticket + 256;
    return t;
}
// What one workgroup ends in one launch.
static bool one_group(int64_t N, int E) { return N * E <= FTK_ROUTE_GATE_FEW; }

}  // namespace ftk

using namespace ftk;

extern "C" {

size_t ftk_route_gate_workspace_bytes(int64_t N, int32_t E)
{
    if (N < 0 || N > 0x7fffffffLL || E < 1 || E > GATE_MAX_EXPERTS) {
        set_error("need 0 <= N < 2^31, 1 <= E <= %d (got N=%lld E=%d)", GATE_MAX_EXPERTS, (long long)N, E);
        return 0;
    }
    return one_group(N, E) ? 256 : gate_table(N < GATE_MAX_GROUPS ? N : GATE_MAX_GROUPS, E).total;
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
    const bool one = one_group(N, E);
    if (!one) FTK_TRY(check_workspace(workspace, workspace_bytes, ftk_route_gate_workspace_bytes(N, E)));
    FTK_TRY(check_device());
    hipStream_t st = (hipStream_t)hip_stream;
    GateArgs a{logits, ldz, N, E, k, normalise != 0, labels, weights, lse, counts, probs, loss, nullptr, nullptr, nullptr};
    if (N == 0) a.ldz = 0;
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return with_share<T, false>(E, k, [&](auto lanes, auto pieces) {
            constexpr int L = decltype(lanes)::value, NP = decltype(pieces)::value;
            constexpr int WAVES = GATE_WAVES<T, L, NP>;
            const size_t lds = align_up((size_t)((L > 64 ? 3 : WAVES + 1) * E + 1) * 4 + 8 * WAVES, 16);
            const int64_t most = L <= 64 ? 256 : GATE_MAX_GROUPS;  // four waves a SIMD, or two that have many registers
            int64_t groups = ceil_div(N, 64 * WAVES / L);
            groups = one ? 1 : groups < most ? groups : most;
            double *parts = nullptr;
            if (!one) {
                const GateTable t = gate_table(groups, E);
                a.sums = (float *)((uint8_t *)workspace + t.sums);
                a.slots = (int32_t *)((uint8_t *)workspace + t.slots);
                a.ticket = (int32_t *)((uint8_t *)workspace + t.ticket);
                parts = (double *)((uint8_t *)workspace + t.parts);
            }
            auto go = [&](auto room) {
                constexpr int K = decltype(room)::value;
                FTK_TRY(allow_lds<((L > 64 ? 3 : WAVES + 1) * L * NP * PIECE<T> + 1) * 4 + 8 * WAVES + 16>((const void *)gate_kernel<T, L, NP, K>));
                gate_kernel<T, L, NP, K><<<(unsigned)groups, 64 * WAVES, lds, st>>>(a);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            };
            if constexpr (sizeof(T) == 2) {
                FTK_TRY(k <= 2 ? go(std::integral_constant<int, 2>{}) : k <= 8 && L >= 8 ? go(std::integral_constant<int, L >= 8 ? 8 : 0>{})
                                                                                         : go(std::integral_constant<int, 0>{}));
            } else {
                FTK_TRY(go(std::integral_constant<int, 0>{}));
            }
            if (!one) {
                gate_end_kernel<<<(unsigned)ceil_div(E, GATE_END_EXPERTS), GATE_END_THREADS, 0, st>>>(a, (int)groups, parts);
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
        return with_share<T, true>(E, k, [&](auto lanes, auto pieces) {
            constexpr int L = decltype(lanes)::value, NP = decltype(pieces)::value;
            const int64_t groups = ceil_div(N, 64 * GATE_GRAD_WAVES / L);
            constexpr size_t lds = (size_t)GATE_GRAD_WAVES * 64 * NP * PIECE<T> * 4;  // a row of each group's
            FTK_TRY(allow_lds<lds>((const void *)gate_grad_kernel<T, L, NP>));
            gate_grad_kernel<T, L, NP><<<(unsigned)(groups < 1024 ? groups : 1024), 64 * GATE_GRAD_WAVES, lds, (hipStream_t)hip_stream>>>(a);
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
    });
}

}  // extern "C"
