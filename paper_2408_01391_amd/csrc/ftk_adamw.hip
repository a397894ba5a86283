// AdamW over many tensors at once, with states in 32 bits or in 8.
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2      (every product and sum rounded to 32 bits)
//   p' = p - lr (wd p + m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps))
//
// One pass: every byte is read and written once, and memory is the bound.  A workgroup has a run of ADAMW_CHUNK elements of one
// tensor, a lane eight consecutive ones at a time; the tensors' addresses travel as the kernel's arguments, so that a call
// needs no table in device memory and nothing waits for one.
// 50 M bf16 weights with 32-bit states and masters, 30 bytes an element: three launches (as many tensors as the arguments hold) of together
// 314 us, 4.8 TB/s; 134 M with 8-bit states, 10 bytes: 290 to 308 us, 4.4 to 4.6 TB/s; a copy reaches 5.0.
//
// 8-bit states (ftkmeans.h has the format): the lanes that have a block of 32 exchange its largest magnitude.
#include <math.h>

#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

constexpr int ADAMW_THREADS = 256, ADAMW_STEP = 8 * ADAMW_THREADS, ADAMW_CHUNK = 4 * ADAMW_STEP;
// The square root's and the reciprocal's instructions take what lies below the normal numbers for 0, roots below 1.1e-19 that is: of no
// weight beside an eps of this size or more, 1.1e-19 / 2e-12 being a step of 32 bits.  Below it both go the longer, exact way.
constexpr float ADAMW_EPS = 2e-12f;
constexpr int64_t ADAMW_MAX = 1LL << 37;  // elements of a tensor: a launch's chunks are 32-bit numbers

// The tensors of a launch: as many as a kernel's arguments of 4 KB hold addresses of.
// (with 8 bits the scales of both states come next, a master last; FIELD_PARAM and FIELD_GRAD are the results of what reads states)
enum { FIELD_PARAM, FIELD_GRAD, FIELD_M, FIELD_V };
template <int FIELDS>
struct AdamwList {
    static constexpr int TENSORS = (4096 - 96) / (FIELDS * 8 + 16);
    void *p[TENSORS][FIELDS];
    int64_t count[TENSORS];
    int32_t first[TENSORS];  // first chunk of a tensor
    int32_t place[TENSORS];  // its place in the caller's list
    int32_t n;
};
struct AdamwRates {
    float b1, b1c, b2, b2c, log_b1, log_b2, lr, eps, decay;
    const float *lr_scale, *grad_scale;
    const int64_t *step;
    uint64_t seed;
};
template <int BITS, bool MASTER>
struct AdamwArgs : AdamwList<4 + (BITS == 8 ? 2 : 0) + MASTER>, AdamwRates {};
static_assert(sizeof(AdamwArgs<8, true>) <= 4096 && sizeof(AdamwArgs<32, false>) <= 4096, "a kernel's arguments hold 4 KB");

// (the key of a tensor at a step: SplitMix64)
constexpr uint64_t GOLDEN = 0x9E3779B97F4A7C15ull;
__device__ __forceinline__ uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
// 32 random bits of an element: a multiplicative hash whose constants were chosen by the flips of its output bits.
__device__ __forceinline__ uint32_t random32(uint32_t key, uint32_t i)
{
    uint32_t x = i ^ key;
    x = (x ^ (x >> 16)) * 0xC8E1ED59u;
    x = (x ^ (x >> 15)) * 0x876BA2B3u;
    return x ^ (x >> 16);
}

// The bits of a code, moved to the top of a 32-bit number's exponent field and of its mantissa, are the number of units it stands for,
// times 2^(-126 - M): e = 0, the code without a leading bit, is what the hardware takes for a number without one, too.
// So a code becomes a number by a product with a power of two, and a number a code by a product that brings it there and a
// cut, at which the random bits below the code have carried into it.  The powers are 2^(126 + M + s) and its inverse, for the
// scale byte s + 127; where that leaves the range of exponents (blocks of numbers above 2^15) a second factor makes up for it.
template <int M>
struct BlockScale {
    static constexpr uint32_t LIMIT = 128 - M;  // the largest scale byte that one factor is enough for (encoding: the least it is not)
    static __device__ __forceinline__ float decode(uint32_t scale)
    {
        return __uint_as_float(scale == 255 ? 0x7fc00000u : min(scale + 126 + M, 254u) << 23);
    }
    static __device__ __forceinline__ float decode_more(uint32_t scale)
    {
        return __uint_as_float((127 + (scale > LIMIT ? scale - LIMIT : 0)) << 23);
    }
    static __device__ __forceinline__ float encode(uint32_t scale) { return __uint_as_float((scale < LIMIT ? LIMIT - scale : 1) << 23); }
    static __device__ __forceinline__ float encode_more(uint32_t scale)
    {
        return __uint_as_float((127 - (scale < LIMIT ? 0 : scale - LIMIT + 1)) << 23);
    }
};
// code e of four in a word, as such a number (M = 3: with its sign)
template <int M>
__device__ __forceinline__ float code_bits(uint32_t word, int e)
{
    if constexpr (M == 3) return __uint_as_float((uint32_t)((int32_t)(word << (24 - 8 * e)) >> 4) & 0x87f00000u);
    else return __uint_as_float((word >> (8 * e) & 255) << 19);
}
// the code of a number of units times 2^(-126 - M), in the top byte
__device__ __forceinline__ uint32_t code_of_signed(float units, uint32_t random)
{
    const uint32_t t = __float_as_uint(units) + (__builtin_amdgcn_ubfe(random, 16, 16) << 4);
    return (t << 4 & 0x7fffffffu) | (t & 0x80000000u);
}
__device__ __forceinline__ uint32_t code_of_positive(float units, float x, uint32_t random)
{
    const uint32_t t = __float_as_uint(units) + ((random & 0xffffu) << 3), least = max(t, 1u << 19);
    return (x > 0.f ? least : t) << 5;  // (a positive number is never rounded to 0)
}
// the scale byte of a block from the largest magnitude's bits
template <int M>
__device__ __forceinline__ uint32_t scale_of(uint32_t max_bits, uint32_t &top)
{
    top = (max_bits + ((1u << (23 - M)) - 1)) >> 23;
    return top > M + 14 ? top - (M + 14) : 0;
}
// the top bytes of four words in one
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0703u), __builtin_amdgcn_perm(b, a, 0x0c0c0703u), 0x05040100u);
}

// E consecutive elements at element alignment, the first n of them, zeros behind.
template <typename T, int E>
struct Some {
    T v[E];
};
template <int E, typename T>
__device__ __forceinline__ Some<T, E> load_some(const T *p, int n)
{
    constexpr int V = E * sizeof(T) > 16 ? 16 / sizeof(T) : E;
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    Some<T, E> r;
    if (n >= E) {
#pragma unroll
        for (int k = 0; k < E; k += V) {
            const vec a = *reinterpret_cast<const vec *>(p + k);
#pragma unroll
            for (int e = 0; e < V; ++e) r.v[k + e] = a[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) r.v[e] = e < n ? p[e] : (T)0;
    }
    return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_some(T *p, const Some<T, E> &r, int n)
{
    constexpr int V = E * sizeof(T) > 16 ? 16 / sizeof(T) : E;
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (n >= E) {
#pragma unroll
        for (int k = 0; k < E; k += V) {
            vec a;
#pragma unroll
            for (int e = 0; e < V; ++e) a[e] = r.v[k + e];
            *reinterpret_cast<vec *>(p + k) = a;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) p[e] = r.v[e];
    }
}
// E codes, four to a word.
template <int E>
__device__ __forceinline__ Some<uint32_t, E / 4> load_codes(const uint8_t *p, int n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    Some<uint32_t, E / 4> r;
#pragma unroll
    for (int k = 0; k < E / 4; ++k) r.v[k] = 0;
    if (n >= E) {
#pragma unroll
        for (int k = 0; k < E / 4; ++k) r.v[k] = *reinterpret_cast<const word *>(p + 4 * k);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) r.v[e / 4] |= (uint32_t)p[e] << (8 * (e % 4));
    }
    return r;
}
template <int E>
__device__ __forceinline__ void store_codes(uint8_t *p, const Some<uint32_t, E / 4> &r, int n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (n >= E) {
#pragma unroll
        for (int k = 0; k < E / 4; ++k) *reinterpret_cast<word *>(p + 4 * k) = r.v[k];
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) p[e] = (uint8_t)(r.v[e / 4] >> (8 * (e % 4)));
    }
}

// What a lane reads of a tensor from element i on.
template <typename P, typename G, int BITS, bool MASTER, int E>
struct AdamwIn {
    static constexpr int FIELDS = 4 + (BITS == 8 ? 2 : 0) + MASTER;
    Some<std::conditional_t<MASTER, float, P>, E> p;
    Some<G, E> g;
    std::conditional_t<BITS == 8, Some<uint32_t, E / 4>, Some<float, E>> m, v;
    uint32_t ms, vs;
    __device__ __forceinline__ void load(void *const *t, int64_t i, int64_t count)
    {
        const int n = (int)min((int64_t)E, count - i);
        ms = vs = 0;
        if (n <= 0) {
            p = {};
            g = {};
            m = {};
            v = {};
            return;
        }
        p = load_some<E>((const std::conditional_t<MASTER, float, P> *)t[MASTER ? FIELDS - 1 : FIELD_PARAM] + i, n);
        g = load_some<E>((const G *)t[FIELD_GRAD] + i, n);
        if constexpr (BITS == 8) {
            m = load_codes<E>((const uint8_t *)t[FIELD_M] + i, n);
            v = load_codes<E>((const uint8_t *)t[FIELD_V] + i, n);
            ms = ((const uint8_t *)t[4])[i >> 5];
            vs = ((const uint8_t *)t[5])[i >> 5];
        } else {
            m = load_some<E>((const float *)t[FIELD_M] + i, n);
            v = load_some<E>((const float *)t[FIELD_V] + i, n);
        }
    }
};

// The chunk's tensor, by halves.
__device__ __forceinline__ int tensor_of(const int32_t *first, int n, int chunk)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Largest over the lanes that have a block of 32, E elements each.
template <int E>
__device__ __forceinline__ uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));                       // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));                       // lane ^ 2
    if constexpr (E == 4) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));  // the other four of eight
    return v;
}

struct AdamwStep {
    float b1, b1c, b2, b2c, rate, vc, eps, decay, gs;
    bool scaled;
    uint32_t key;
};

// E consecutive elements of a lane, n of them there (E, where all are).
template <typename P, typename G, int BITS, bool MASTER, int E>
__device__ __forceinline__ void adamw_some(const AdamwIn<P, G, BITS, MASTER, E> &in, const AdamwStep &a, void *const *t, int64_t i, int n)
{
    using M3 = BlockScale<3>;
    using M4 = BlockScale<4>;
    float m[E], v[E];
    {
#pragma clang fp contract(off)
        // (a power of two with b1 does not change how the product is rounded)
        float mf = a.b1, vf = a.b2;
        if constexpr (BITS == 8) {
            mf = a.b1 * M3::decode(in.ms);
            vf = a.b2 * M4::decode(in.vs);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (BITS == 8) {
                m[e] = mf * code_bits<3>(in.m.v[e / 4], e % 4);
                v[e] = vf * code_bits<4>(in.v.v[e / 4], e % 4);
            } else {
                m[e] = mf * in.m.v[e];
                v[e] = vf * in.v.v[e];
            }
        }
        if constexpr (BITS == 8) {
            if (__any(in.ms > M3::LIMIT || in.vs > M4::LIMIT)) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    m[e] = m[e] * M3::decode_more(in.ms);
                    v[e] = v[e] * M4::decode_more(in.vs);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float g = (float)in.g.v[e];
            if (a.scaled) g = g * a.gs;
            m[e] = m[e] + a.b1c * g;
            const float gg = g * g;
            v[e] = v[e] + a.b2c * gg;
        }
    }
    Some<float, E> p;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float ratio;
        if (a.eps < ADAMW_EPS) ratio = m[e] / (sqrtf(v[e]) * sqrtf(a.vc) + a.eps);
        else ratio = m[e] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e] * a.vc) + a.eps);
        // (the decay joins the update before the weight: 1 - lr decay would be rounded to a multiple of 2^-24, for all weights alike)
        const float w = (float)in.p.v[e];
        p.v[e] = w - fmaf(a.decay, w, a.rate * ratio);
        // (the 16-bit weight is the master rounded; an instruction that adds and rounds to 16 bits at once would take the unrounded sum)
        if constexpr (MASTER) asm("" : "+v"(p.v[e]));
    }
    if (n > 0) {
        if constexpr (MASTER) store_some((float *)t[in.FIELDS - 1] + i, p, n);
        Some<P, E> o;
#pragma unroll
        for (int e = 0; e < E; ++e) o.v[e] = (P)p.v[e];
        store_some((P *)t[FIELD_PARAM] + i, o, n);
    }
    if constexpr (BITS == 8) {
        // (elements behind the last one are zeros; v has no sign, but a NaN may)
        uint32_t mt = 0, vt = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            mt = max(mt, mag_bits(m[e]));
            vt = max(vt, mag_bits(v[e]));
        }
        uint32_t mtop, vtop;
        const uint32_t ms = scale_of<3>(block_max<E>(mt), mtop), vs = scale_of<4>(block_max<E>(vt), vtop);
        const float mu = M3::encode(ms), vu = M4::encode(vs);
        const bool wide = __any(ms >= M3::LIMIT || vs >= M4::LIMIT);
        Some<uint32_t, E / 4> mo, vo;
#pragma unroll
        for (int k = 0; k < E / 4; ++k) {
            uint32_t mc[4], vcode[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = m[4 * k + e], y = v[4 * k + e];
                if (wide) {
                    x *= M3::encode_more(ms);
                    y *= M4::encode_more(vs);
                }
                const uint32_t r = random32(a.key, (uint32_t)i | (4 * k + e));
                mc[e] = code_of_signed(x * mu, r);
                vcode[e] = code_of_positive(y * vu, y, r);
            }
            mo.v[k] = top_bytes(mc[0], mc[1], mc[2], mc[3]);
            vo.v[k] = top_bytes(vcode[0], vcode[1], vcode[2], vcode[3]);
        }
        if (n > 0) {
            store_codes<E>((uint8_t *)t[FIELD_M] + i, mo, n);
            store_codes<E>((uint8_t *)t[FIELD_V] + i, vo, n);
            if ((threadIdx.x & (32 / E - 1)) == 0) {
                ((uint8_t *)t[4])[i >> 5] = mtop >= 255 ? 255 : (uint8_t)ms;
                ((uint8_t *)t[5])[i >> 5] = vtop >= 255 ? 255 : (uint8_t)vs;
            }
        }
    } else if (n > 0) {
        Some<float, E> mo, vo;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            mo.v[e] = m[e];
            vo.v[e] = v[e];
        }
        store_some((float *)t[FIELD_M] + i, mo, n);
        store_some((float *)t[FIELD_V] + i, vo, n);
    }
}

template <typename P, typename G, int BITS, bool MASTER, int E>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwArgs<BITS, MASTER> a)
{
    using In = AdamwIn<P, G, BITS, MASTER, E>;
    constexpr int STEP = E * ADAMW_THREADS;
    const int which = tensor_of(a.first, a.n, (int)blockIdx.x);
    void *const *const t = a.p[which];
    const int64_t count = a.count[which], from = (int64_t)((int)blockIdx.x - a.first[which]) * ADAMW_CHUNK;
    int64_t i = from + threadIdx.x * E;
    In in[2];
    in[0].load(t, i, count);
    const int64_t step = max((int64_t)1, *a.step);
    const float c1 = -expm1f((float)step * a.log_b1), c2 = -expm1f((float)step * a.log_b2);
    const float lr = a.lr_scale ? a.lr * *a.lr_scale : a.lr;
    AdamwStep s{a.b1, a.b1c, a.b2, a.b2c, lr / c1, 1.f / c2, a.eps, lr * a.decay, a.grad_scale ? *a.grad_scale : 1.f, a.grad_scale != nullptr, 0};
    if constexpr (BITS == 8)
        s.key = (uint32_t)mix64(mix64(mix64(a.seed + GOLDEN * (uint64_t)step) + (uint64_t)a.place[which]) + (uint64_t)(from >> 32));
    if (from + ADAMW_CHUNK <= count) {
        // (a chunk with all its elements: no bounds, and the next ones are requested a step ahead)
#pragma unroll
        for (int k = 0; k < ADAMW_CHUNK / STEP; ++k, i += STEP) {
            if (k + 1 < ADAMW_CHUNK / STEP) in[(k + 1) & 1].load(t, i + STEP, i + STEP + E);
            adamw_some(in[k & 1], s, t, i, E);
        }
        return;
    }
    const int64_t end = min(from + ADAMW_CHUNK, count);
    for (int64_t at = from; at < end; at += STEP, i += STEP) {
        if (at > from) in[0].load(t, i, count);
        adamw_some(in[0], s, t, i, (int)min((int64_t)E, count - i));
    }
}

template <typename T>
__global__ __launch_bounds__(ADAMW_THREADS) void moments_kernel(const AdamwList<6> a)
{
    const int which = tensor_of(a.first, a.n, (int)blockIdx.x);
    void *const *const t = a.p[which];
    const int64_t count = a.count[which], from = (int64_t)((int)blockIdx.x - a.first[which]) * ADAMW_CHUNK;
    const int64_t end = min(from + ADAMW_CHUNK, count);
#pragma unroll 2
    for (int64_t i = from + threadIdx.x * 8; i < end; i += ADAMW_STEP) {
        const int n = (int)min((int64_t)8, count - i);
        const Some<uint32_t, 2> m = load_codes<8>((const uint8_t *)t[FIELD_M] + i, n), v = load_codes<8>((const uint8_t *)t[FIELD_V] + i, n);
        const uint32_t ms = ((const uint8_t *)t[4])[i >> 5], vs = ((const uint8_t *)t[5])[i >> 5];
        const float mf = BlockScale<3>::decode(ms), vf = BlockScale<4>::decode(vs), mw = BlockScale<3>::decode_more(ms),
                    vw = BlockScale<4>::decode_more(vs);
        Some<T, 8> mo, vo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mo.v[e] = (T)(code_bits<3>(m.v[e / 4], e % 4) * mf * mw);
            vo.v[e] = (T)(code_bits<4>(v.v[e / 4], e % 4) * vf * vw);
        }
        store_some((T *)t[FIELD_PARAM] + i, mo, n);
        store_some((T *)t[FIELD_GRAD] + i, vo, n);
    }
}

// Launches for the tensors that take part, as many at a time as the arguments hold: fields(addresses, place) for each.
template <int FIELDS, typename Takes, typename Fields, typename Launch>
static ftk_status by_launches(AdamwList<FIELDS> &a, const ftk_adamw_tensor *tensors, int n, Takes &&takes, Fields &&fields, Launch &&launch)
{
    int64_t chunks = 0;
    a.n = 0;
    for (int i = 0; i < n; ++i) {
        if (!takes(tensors[i])) continue;
        a.first[a.n] = (int32_t)chunks;
        a.place[a.n] = i;
        a.count[a.n] = tensors[i].count;
        fields(a.p[a.n++], i);
        chunks += ceil_div(tensors[i].count, ADAMW_CHUNK);
        if (a.n < a.TENSORS) continue;
        FTK_TRY(launch((unsigned)chunks));
        chunks = 0;
        a.n = 0;
    }
    return a.n ? launch((unsigned)chunks) : FTK_OK;
}

// What a list's tensors need; `params`: whether weights and gradients do.
static ftk_status check_tensors(const ftk_adamw_tensor *tensors, int32_t n, int32_t bits, bool params, ftk_dtype dtype,
                                ftk_dtype grad_dtype)
{
    if (n < 0 || (n > 0 && !tensors)) {
        set_error("need a list of n >= 0 tensors (got n=%d)", n);
        return FTK_EINVAL;
    }
    int masters = -1;
    for (int i = 0; i < n; ++i) {
        const ftk_adamw_tensor &t = tensors[i];
        if (t.count < 0 || t.count > ADAMW_MAX) {
            set_error("tensor %d: need 0 <= count <= 2^37 (got %lld)", i, (long long)t.count);
            return FTK_EINVAL;
        }
        if (t.count == 0 || (params && !t.grad)) continue;
        FTK_TRY(check_ptr(t.m, bits == 8 ? 1 : 4, "m"));
        FTK_TRY(check_ptr(t.v, bits == 8 ? 1 : 4, "v"));
        if (bits == 8) {
            FTK_TRY(check_ptr(t.m_scales, 1, "m_scales"));
            FTK_TRY(check_ptr(t.v_scales, 1, "v_scales"));
        }
        if (!params) continue;
        FTK_TRY(check_ptr(t.param, dtype_size(dtype), "param"));
        FTK_TRY(check_ptr(t.grad, dtype_size(grad_dtype), "grad"));
        if (t.master) FTK_TRY(check_ptr(t.master, 4, "master"));
        if (masters >= 0 && masters != (t.master != nullptr)) {
            set_error("tensor %d: either all tensors of a call have a master or none", i);
            return FTK_EINVAL;
        }
        masters = t.master != nullptr;
    }
    if (masters == 1 && dtype == FTK_F32) {
        set_error("weights in 32 bits are their own masters");
        return FTK_EINVAL;
    }
    return FTK_OK;
}

template <typename P, typename G, int BITS, bool MASTER>
static ftk_status launch_adamw(const AdamwRates &rates, const ftk_adamw_tensor *tensors, int n, hipStream_t st)
{
    AdamwArgs<BITS, MASTER> a;
    static_cast<AdamwRates &>(a) = rates;
    return by_launches(
        a, tensors, n, [](const ftk_adamw_tensor &t) { return t.count > 0 && t.grad; },
        [&](void **p, int i) {
            const ftk_adamw_tensor &t = tensors[i];
            p[FIELD_PARAM] = t.param;
            p[FIELD_GRAD] = const_cast<void *>(t.grad);
            p[FIELD_M] = t.m;
            p[FIELD_V] = t.v;
            if constexpr (BITS == 8) {
                p[4] = t.m_scales;
                p[5] = t.v_scales;
            }
            if constexpr (MASTER) p[BITS == 8 ? 6 : 4] = t.master;
        },
        [&](unsigned chunks) {
            adamw_kernel<P, G, BITS, MASTER, BITS == 8 ? 8 : 4><<<chunks, ADAMW_THREADS, 0, st>>>(a);
            FTK_TRY_HIP(hipGetLastError());
            return FTK_OK;
        });
}

}  // namespace ftk

using namespace ftk;

extern "C" {

ftk_status ftk_adamw_step(ftk_dtype dtype, ftk_dtype grad_dtype, int32_t state_bits, const ftk_adamw_tensor *tensors, int32_t n,
                          const ftk_adamw_options *options, void *hip_stream)
{
    FTK_TRY(check_mx_type(dtype));
    FTK_TRY(check_mx_type(grad_dtype));
    if (dtype != FTK_F32 && grad_dtype != FTK_F32 && grad_dtype != dtype) {
        set_error("gradients of 16-bit weights come in their type or in 32 bits");
        return FTK_EINVAL;
    }
    if (state_bits != 8 && state_bits != 32) {
        set_error("states have 8 or 32 bits (got %d)", state_bits);
        return FTK_EINVAL;
    }
    if (!options) {
        set_error("options is NULL");
        return FTK_EINVAL;
    }
    const ftk_adamw_options &o = *options;
    if (!(o.beta1 >= 0 && o.beta1 < 1 && o.beta2 >= 0 && o.beta2 < 1 && o.eps >= 0 && o.weight_decay >= 0) || !isfinite(o.lr) ||
        !isfinite(o.eps) || !isfinite(o.weight_decay)) {
        set_error("need a finite lr, 0 <= beta1, beta2 < 1, finite eps and weight_decay >= 0 (got %g, %g, %g, %g, %g)", o.lr, o.beta1,
                  o.beta2, o.eps, o.weight_decay);
        return FTK_EINVAL;
    }
    FTK_TRY(check_ptr(o.step, 8, "step"));
    if (o.lr_scale) FTK_TRY(check_ptr(o.lr_scale, 4, "lr_scale"));
    if (o.grad_scale) FTK_TRY(check_ptr(o.grad_scale, 4, "grad_scale"));
    FTK_TRY(check_tensors(tensors, n, state_bits, true, dtype, grad_dtype));
    FTK_TRY(check_device());
    bool master = false;
    for (int i = 0; i < n; ++i) master |= tensors[i].count > 0 && tensors[i].grad && tensors[i].master;
    AdamwRates a;
    a.b1 = (float)o.beta1;
    a.b1c = (float)(1 - o.beta1);
    a.b2 = (float)o.beta2;
    a.b2c = (float)(1 - o.beta2);
    a.log_b1 = (float)log(o.beta1);
    a.log_b2 = (float)log(o.beta2);
    a.lr = (float)o.lr;
    a.eps = (float)o.eps;
    a.decay = (float)o.weight_decay;
    a.lr_scale = o.lr_scale;
    a.grad_scale = o.grad_scale;
    a.step = o.step;
    a.seed = o.seed;
    hipStream_t st = (hipStream_t)hip_stream;
    auto with_bits = [&](auto p, auto g, auto m) {
        using P = typename decltype(p)::type;
        using G = typename decltype(g)::type;
        constexpr bool M = decltype(m)::value;
        return state_bits == 8 ? launch_adamw<P, G, 8, M>(a, tensors, n, st) : launch_adamw<P, G, 32, M>(a, tensors, n, st);
    };
    if (dtype == FTK_F32)
        return with_mx_type(grad_dtype, [&](auto g) { return with_bits(TypeTag<float>{}, g, std::false_type{}); });
    auto with_master = [&](auto p, auto g) { return master ? with_bits(p, g, std::true_type{}) : with_bits(p, g, std::false_type{}); };
    auto with_grads = [&](auto p) { return grad_dtype == FTK_F32 ? with_master(p, TypeTag<float>{}) : with_master(p, p); };
    return dtype == FTK_BF16 ? with_grads(TypeTag<__bf16>{}) : with_grads(TypeTag<_Float16>{});
}

ftk_status ftk_adamw_moments(ftk_dtype dtype, const ftk_adamw_tensor *tensors, int32_t n, void *const *m_out, void *const *v_out,
                             void *hip_stream)
{
    FTK_TRY(check_mx_type(dtype));
    FTK_TRY(check_tensors(tensors, n, 8, false, dtype, dtype));
    if (n > 0 && (!m_out || !v_out)) {
        set_error("m_out or v_out is NULL");
        return FTK_EINVAL;
    }
    for (int i = 0; i < n; ++i)
        if (tensors[i].count > 0) {
            FTK_TRY(check_ptr(m_out[i], dtype_size(dtype), "m_out"));
            FTK_TRY(check_ptr(v_out[i], dtype_size(dtype), "v_out"));
        }
    FTK_TRY(check_device());
    AdamwList<6> a;
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return by_launches(
            a, tensors, n, [](const ftk_adamw_tensor &t) { return t.count > 0; },
            [&](void **p, int i) {
                const ftk_adamw_tensor &t = tensors[i];
                p[FIELD_PARAM] = m_out[i];
                p[FIELD_GRAD] = v_out[i];
                p[FIELD_M] = t.m;
                p[FIELD_V] = t.v;
                p[4] = t.m_scales;
                p[5] = t.v_scales;
            },
            [&](unsigned chunks) {
                moments_kernel<T><<<chunks, ADAMW_THREADS, 0, (hipStream_t)hip_stream>>>(a);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            });
    });
}

}  // extern "C"
