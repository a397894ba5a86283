// AdamW over many tensors at once, with states in 32 bits or in 8.
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2      (every product and sum rounded to 32 bits)
//   p' = p - lr (wd p + m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps))
//
// One pass: every byte is read and written once, and memory is the bound.  A workgroup has a run of ADAMW_CHUNK elements of one
// tensor, a lane eight consecutive ones at a time; the tensors' addresses travel as the kernel's arguments, so that a call
// needs no table in device memory and nothing waits for one.
//
// 8-bit states (ftkmeans.h has the format): four lanes have a block of 32, whose largest magnitude they exchange.  Codes are
// made from the bits of the 32-bit number: in units of the block's scale the exponent field and the first M bits behind
// it are the code, but for a constant; random bits are added below them before the rest is cut off.  Numbers
// below the first binade get 2^M added first, which puts their bits in the same place.
#include <math.h>

#include "ftk_mx4.h"
#include "ftk_quads.h"

namespace ftk {

constexpr int ADAMW_THREADS = 256, ADAMW_EACH = 8, ADAMW_STEP = ADAMW_THREADS * ADAMW_EACH, ADAMW_CHUNK = 4 * ADAMW_STEP;
constexpr int ADAMW_TENSORS = 52;  // of a launch: a kernel's arguments hold 4 KB
constexpr int64_t ADAMW_MAX = 1LL << 37;  // elements of a tensor: a launch's chunks are 32-bit numbers

struct AdamwArgs {
    ftk_adamw_tensor t[ADAMW_TENSORS];
    int32_t first[ADAMW_TENSORS];  // first chunk of a tensor
    int32_t place[ADAMW_TENSORS];  // its place in the caller's list
    int32_t n;
    float b1, b1c, b2, b2c, log_b1, log_b2, lr, eps, decay;
    const float *lr_scale, *grad_scale;
    const int64_t *step;
    uint64_t seed;
};
static_assert(sizeof(AdamwArgs) <= 4096, "a kernel's arguments hold 4 KB");

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

// 2^(M + s) for the scale byte s + 127, NaN for 255; see decode8.
template <int M>
__device__ __forceinline__ float decode_factor(uint32_t scale)
{
    return __uint_as_float(scale == 255 ? 0x7fc00000u : min(scale + M, 254u) << 23);
}
// A code as the bits of a 32-bit number is its number of units times 2^(-126 - M).
template <int M>
__device__ __forceinline__ float decode8(uint32_t code, float factor)
{
    const float size = __uint_as_float((code & ((16u << M) - 1)) << (23 - M)) * 0x1p126f * factor;
    return M == 3 && (code & 128) ? -size : size;
}
template <int M>
__device__ __forceinline__ uint32_t scale_of(uint32_t max_bits, uint32_t &top)
{
    top = (max_bits + ((1u << (23 - M)) - 1)) >> 23;
    return top > M + 14 ? top - (M + 14) : 0;
}
template <int M>
__device__ __forceinline__ uint32_t encode8(float x, float per_unit, uint32_t random)
{
    const float y = fabsf(x) * per_unit;
    const bool low = y < (float)(1 << M);
    const float t = low ? y + (float)(1 << M) : y;
    uint32_t code = ((__float_as_uint(t) + random) >> (23 - M)) - ((126u + M) << M) - (low ? 1u << M : 0u);
    if (M == 3) return (code & 127) | (__float_as_uint(x) >> 31) << 7;
    if (x > 0.f) code = max(code, 1u);
    return code & 255;
}

// Eight consecutive elements at element alignment, the first n of them.
template <typename T>
struct Eight {
    T v[8];
};
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *p, int n)
{
    typedef T vec __attribute__((ext_vector_type(sizeof(T) == 4 ? 4 : 8), aligned(sizeof(T))));
    Eight<T> r;
    if (n >= 8) {
        if constexpr (sizeof(T) == 4) {
            const vec a = *reinterpret_cast<const vec *>(p), b = *reinterpret_cast<const vec *>(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                r.v[e] = a[e];
                r.v[4 + e] = b[e];
            }
        } else {
            const vec a = *reinterpret_cast<const vec *>(p);
#pragma unroll
            for (int e = 0; e < 8; ++e) r.v[e] = a[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = e < n ? p[e] : (T)0;
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_eight(T *p, const Eight<T> &r, int n)
{
    typedef T vec __attribute__((ext_vector_type(sizeof(T) == 4 ? 4 : 8), aligned(sizeof(T))));
    if (n >= 8) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<vec *>(p) = vec{r.v[0], r.v[1], r.v[2], r.v[3]};
            *reinterpret_cast<vec *>(p + 4) = vec{r.v[4], r.v[5], r.v[6], r.v[7]};
        } else {
            *reinterpret_cast<vec *>(p) = vec{r.v[0], r.v[1], r.v[2], r.v[3], r.v[4], r.v[5], r.v[6], r.v[7]};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = r.v[e];
    }
}

template <typename P, typename G, int BITS, bool MASTER>
struct AdamwIn {
    using S = std::conditional_t<BITS == 8, uint8_t, float>;
    Eight<std::conditional_t<MASTER, float, P>> p;
    Eight<G> g;
    Eight<S> m, v;
    uint32_t ms, vs;
    __device__ __forceinline__ void load(const ftk_adamw_tensor &t, int64_t i)
    {
        const int n = (int)min((int64_t)8, t.count - i);
        ms = vs = 0;
        if (n <= 0) {
            p = {};
            g = {};
            m = {};
            v = {};
            return;
        }
        if constexpr (MASTER) p = load_eight(t.master + i, n);
        else p = load_eight((const P *)t.param + i, n);
        g = load_eight((const G *)t.grad + i, n);
        m = load_eight((const S *)t.m + i, n);
        v = load_eight((const S *)t.v + i, n);
        if constexpr (BITS == 8) {
            ms = t.m_scales[i >> 5];
            vs = t.v_scales[i >> 5];
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

template <typename P, typename G, int BITS, bool MASTER>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwArgs a)
{
    using In = AdamwIn<P, G, BITS, MASTER>;
    const int which = tensor_of(a.first, a.n, (int)blockIdx.x);
    const ftk_adamw_tensor t = a.t[which];
    const int64_t from = (int64_t)((int)blockIdx.x - a.first[which]) * ADAMW_CHUNK;
    const int64_t end = min(from + ADAMW_CHUNK, t.count);
    int64_t i = from + threadIdx.x * ADAMW_EACH;
    In in;
    in.load(t, i);
    const int64_t step = max((int64_t)1, *a.step);
    const float c1 = -expm1f((float)step * a.log_b1), c2 = -expm1f((float)step * a.log_b2);
    const float lr = a.lr_scale ? a.lr * *a.lr_scale : a.lr, gs = a.grad_scale ? *a.grad_scale : 1.f;
    const float rate = lr / c1, vc = 1.f / c2, decay = lr * a.decay;
    uint32_t key = 0;
    if constexpr (BITS == 8)
        key = (uint32_t)mix64(mix64(mix64(a.seed + GOLDEN * (uint64_t)step) + (uint64_t)a.place[which]) + (uint64_t)(from >> 32));
    for (int64_t at = from; at < end; at += ADAMW_STEP, i += ADAMW_STEP) {
        In next;
        next.load(t, at + ADAMW_STEP < end ? i + ADAMW_STEP : t.count);
        const int n = (int)min((int64_t)8, t.count - i);
        float m[8], v[8];
        Eight<float> p;
        float mf = 0.f, vf = 0.f;
        if constexpr (BITS == 8) {
            mf = decode_factor<3>(in.ms);
            vf = decode_factor<4>(in.vs);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma clang fp contract(off)
            if constexpr (BITS == 8) {
                m[e] = decode8<3>(in.m.v[e], mf);
                v[e] = decode8<4>(in.v.v[e], vf);
            } else {
                m[e] = in.m.v[e];
                v[e] = in.v.v[e];
            }
            float g = (float)in.g.v[e];
            if (a.grad_scale) g = g * gs;
            m[e] = a.b1 * m[e] + a.b1c * g;
            const float gg = g * g;
            v[e] = a.b2 * v[e] + a.b2c * gg;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float root = __builtin_amdgcn_sqrtf(v[e] * vc) + a.eps;
            const float w = (float)in.p.v[e];
            p.v[e] = w - decay * w - rate * m[e] * __builtin_amdgcn_rcpf(root);
        }
        if constexpr (BITS == 8) {
            uint32_t mt = 0, vt = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                mt = max(mt, e < n ? mag_bits(m[e]) : 0u);
                vt = max(vt, e < n ? mag_bits(v[e]) : 0u);
            }
            // (the four lanes of a block)
            mt = max(mt, (uint32_t)__builtin_amdgcn_mov_dpp((int)mt, 0xB1, 0xf, 0xf, true));
            vt = max(vt, (uint32_t)__builtin_amdgcn_mov_dpp((int)vt, 0xB1, 0xf, 0xf, true));
            mt = max(mt, (uint32_t)__builtin_amdgcn_mov_dpp((int)mt, 0x4E, 0xf, 0xf, true));
            vt = max(vt, (uint32_t)__builtin_amdgcn_mov_dpp((int)vt, 0x4E, 0xf, 0xf, true));
            uint32_t mtop, vtop;
            const uint32_t ms = scale_of<3>(mt, mtop), vs = scale_of<4>(vt, vtop);
            const float mu = __uint_as_float((254u - ms) << 23), vu = __uint_as_float((254u - vs) << 23);
            Eight<uint8_t> mc, vc8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t r = random32(key, (uint32_t)(i + e));
                mc.v[e] = (uint8_t)encode8<3>(m[e], mu, (r >> 16) << 4);
                vc8.v[e] = (uint8_t)encode8<4>(v[e], vu, (r & 0xffffu) << 3);
            }
            if (n > 0) {
                store_eight((uint8_t *)t.m + i, mc, n);
                store_eight((uint8_t *)t.v + i, vc8, n);
                if ((threadIdx.x & 3) == 0) {
                    t.m_scales[i >> 5] = mtop >= 255 ? 255 : (uint8_t)ms;
                    t.v_scales[i >> 5] = vtop >= 255 ? 255 : (uint8_t)vs;
                }
            }
        } else if (n > 0) {
            Eight<float> ms, vs;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ms.v[e] = m[e];
                vs.v[e] = v[e];
            }
            store_eight((float *)t.m + i, ms, n);
            store_eight((float *)t.v + i, vs, n);
        }
        if (n > 0) {
            if constexpr (MASTER) store_eight(t.master + i, p, n);
            Eight<P> o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o.v[e] = (P)p.v[e];
            store_eight((P *)t.param + i, o, n);
        }
        in = next;
    }
}

struct MomentsArgs {
    struct {
        const uint8_t *m, *v, *m_scales, *v_scales;
        void *m_out, *v_out;
        int64_t count;
    } t[ADAMW_TENSORS];
    int32_t first[ADAMW_TENSORS];
    int32_t n;
};
template <typename T>
__global__ __launch_bounds__(ADAMW_THREADS) void moments_kernel(const MomentsArgs a)
{
    const int which = tensor_of(a.first, a.n, (int)blockIdx.x);
    const auto &t = a.t[which];
    const int64_t from = (int64_t)((int)blockIdx.x - a.first[which]) * ADAMW_CHUNK;
    const int64_t end = min(from + ADAMW_CHUNK, t.count);
#pragma unroll 2
    for (int64_t i = from + threadIdx.x * ADAMW_EACH; i < end; i += ADAMW_STEP) {
        const int n = (int)min((int64_t)8, t.count - i);
        const Eight<uint8_t> m = load_eight(t.m + i, n), v = load_eight(t.v + i, n);
        const float mf = decode_factor<3>(t.m_scales[i >> 5]), vf = decode_factor<4>(t.v_scales[i >> 5]);
        Eight<T> mo, vo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mo.v[e] = (T)decode8<3>(m.v[e], mf);
            vo.v[e] = (T)decode8<4>(v.v[e], vf);
        }
        store_eight((T *)t.m_out + i, mo, n);
        store_eight((T *)t.v_out + i, vo, n);
    }
}

// Launches for the tensors that take part, ADAMW_TENSORS at a time: add(args, slot, place) for each.
template <typename Args, typename Takes, typename Add, typename Launch>
static ftk_status by_launches(Args &a, const ftk_adamw_tensor *tensors, int n, Takes &&takes, Add &&add, Launch &&launch)
{
    int64_t chunks = 0;
    a.n = 0;
    for (int i = 0; i < n; ++i) {
        if (!takes(tensors[i])) continue;
        a.first[a.n] = (int32_t)chunks;
        add(a.n++, i);
        chunks += ceil_div(tensors[i].count, ADAMW_CHUNK);
        if (a.n < ADAMW_TENSORS) continue;
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
static ftk_status launch_adamw(AdamwArgs &a, const ftk_adamw_tensor *tensors, int n, hipStream_t st)
{
    return by_launches(
        a, tensors, n, [](const ftk_adamw_tensor &t) { return t.count > 0 && t.grad; },
        [&](int slot, int i) {
            a.t[slot] = tensors[i];
            a.place[slot] = i;
        },
        [&](unsigned chunks) {
            adamw_kernel<P, G, BITS, MASTER><<<chunks, ADAMW_THREADS, 0, st>>>(a);
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
    AdamwArgs a;
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
    MomentsArgs a;
    return with_mx_type(dtype, [&](auto tag) {
        using T = typename decltype(tag)::type;
        return by_launches(
            a, tensors, n, [](const ftk_adamw_tensor &t) { return t.count > 0; },
            [&](int slot, int i) {
                const ftk_adamw_tensor &t = tensors[i];
                a.t[slot] = {(const uint8_t *)t.m, (const uint8_t *)t.v, t.m_scales, t.v_scales, m_out[i], v_out[i], t.count};
            },
            [&](unsigned chunks) {
                moments_kernel<T><<<chunks, ADAMW_THREADS, 0, (hipStream_t)hip_stream>>>(a);
                FTK_TRY_HIP(hipGetLastError());
                return FTK_OK;
            });
    });
}

}  // extern "C"
