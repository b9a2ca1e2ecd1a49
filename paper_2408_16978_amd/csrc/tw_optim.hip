// What a step does with the gradients (include/fpdt_tokenwise.h): their norm over all tensors, AdamW with states in 32 or
// in 8 bits, and the values of 8-bit states.
//
// All of it is bound by the memory: every array is read or written once.  A launch covers many tensors: their addresses are
// kernel arguments (nothing to copy or to keep on the device, so a call may be captured), their elements are cut into units of
// UNIT, and a workgroup finds its tensor by comparing its unit with the first units of all, one per lane.
#include <cmath>

#include "../../include/fpdt_tokenwise.h"
#include "tw_common.h"

namespace {

using namespace fpdt_tw;

// Elements of a unit: as many as a thread can have under way, where that gives every compute unit four workgroups; a quarter of
// them otherwise (150 tensors of 64 to 65536 elements, 1.4 million in all: three launches of the step 16.3 us for 20.6, the
// norm's 4.2 for 4.8).
constexpr int UNIT = 4096, UNIT8 = 2048, SMALL_UNIT = 1024;  // (8-bit states: 1006 us with 2048, 1034 with 4096, which in 32 bits takes 1281 for 1307)
constexpr int NORM_UNIT = 16384, SMALL_NORM_UNIT = 4096;
constexpr int ENOUGH = 1024;  // units
constexpr int BLOCK = 128;        // elements of a block of 8-bit states
constexpr int MOST_UNITS = (1 << 24) - 1;  // of a launch: fewer than 2^32 lanes

constexpr int64_t MOST_ELEMENTS = (int64_t)UNIT8 * MOST_UNITS;  // of a tensor

// ---- lists of tensors as kernel arguments (at most 4 KB)
template <class Tensor, int N> struct List {
    unsigned first[N];  // unit that the tensor begins with; ~0 behind the last
    Tensor t[N];
};

// The tensor of a unit: how many tensors begin at it or before.
template <int N> __device__ __forceinline__ int find(const unsigned (&first)[N], unsigned unit)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; i += 64) {
        const int k = i + (threadIdx.x & 63);
        n += __popcll(__ballot(k < N && first[k < N ? k : 0] <= unit));
    }
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// `left` elements are left at p; WHOLE: at least V.
template <class T, int V, bool WHOLE> __device__ __forceinline__ Vec<T, V> load_to(const T* p, int64_t left)
{
    if (WHOLE || left >= V) return load_once<V>(p);
    Vec<T, V> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = e < left ? p[e] : T(0);
    return v;
}
template <bool WHOLE, class T, int V> __device__ __forceinline__ void store_to(T* p, int64_t left, const Vec<T, V>& v)
{
    if (WHOLE || left >= V) {
        store_once(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < left) p[e] = v.e[e];
}

// ---- the norm
struct NormTensor {
    const void* g;
    int64_t n;
};
constexpr int NORM_TENSORS = 192, NORM_GROUPS = 1024;
struct NormArgs {
    List<NormTensor, NORM_TENSORS> list;
    double* partial;
    unsigned units;
};

__device__ double group_sum(double v, double* lds)
{
    v = wave_sum_f64(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
    for (unsigned i = 0; i < blockDim.x / 64; ++i) v += lds[i];
    return v;
}

// Squares and sums in 64 bits: no gradient that a float holds overflows or vanishes in them.  A workgroup leaves one
// partial sum, in the same place and of the same units in every call.
template <class T, int U> __global__ __launch_bounds__(256) void grad_norm_kernel(NormArgs a)
{
    constexpr int V = 16 / sizeof(T), N = U / 256 / V;
    __shared__ double lds[4];
    double sum = 0;
    for (unsigned u = blockIdx.x; u < a.units; u += gridDim.x) {
        const int k = find(a.list.first, u);
        const int64_t at = (int64_t)(u - a.list.first[k]) * U, left = a.list.t[k].n - at;
        const T* g = static_cast<const T*>(a.list.t[k].g) + at;
        Vec<T, V> x[N];
        if (left >= U) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = load_once<V>(g + (i * 256 + threadIdx.x) * V);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = (i * 256 + threadIdx.x) * V;
                x[i] = {};
                if (c < left) x[i] = load_to<T, V, false>(g + c, left - c);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double d = to_float(x[i].e[e]);
                sum = fma(d, d, sum);
            }
    }
    sum = group_sum(sum, lds);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm_end_kernel(const double* partial, int n, double max_norm, float* out)
{
    __shared__ double lds[16];
    double sum = 0;
    for (int i = threadIdx.x; i < n; i += 1024) sum += partial[i];
    sum = group_sum(sum, lds);
    if (threadIdx.x) return;
    const double norm = sqrt(sum);
    double c = max_norm / (norm + 1e-6);
    if (c > 1) c = 1;
    out[0] = (float)norm;
    out[1] = isfinite(norm) ? (float)c : NAN;
}

// ---- AdamW
struct Tensor32 {
    float* p;
    uint16_t* w;
    void* g;
    void* m;
    void* v;
    int64_t n;
    double decay;
};
struct Tensor8 : Tensor32 {
    uint8_t *m_exp, *v_exp;
    unsigned ordinal, pad;
};
constexpr int TENSORS32 = 64, TENSORS8 = 47;  // what 4 KB hold

struct AdamwHyper {
    double lr, bc1, bc2, log1, log2;  // bc = 1 - beta^step; logarithms of the betas
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale;
    int64_t step;
    float b1, c1, b2, c2, eps;  // c = 1 - beta
    unsigned seed;
    int zero;
};
template <class Tensor, int N> struct AdamwArgs {
    AdamwHyper h;
    List<Tensor, N> list;
};
static_assert(sizeof(AdamwArgs<Tensor32, TENSORS32>) <= 4096 && sizeof(AdamwArgs<Tensor8, TENSORS8>) <= 4096 && sizeof(NormArgs) <= 4096, "kernel arguments");

// What is the same for all elements of a tensor.
struct Step {
    float keep, rate, root, eps, scale, b1, c1, b2, c2;
    int64_t step;
    bool skip;
};
__device__ __forceinline__ Step make_step(const AdamwHyper& h, double decay)
{
    Step s;
    const double lr = h.lr_dev ? (double)*h.lr_dev : h.lr;
    double bc1 = h.bc1, bc2 = h.bc2;
    s.step = h.step;
    if (h.step_dev) {
        s.step = *h.step_dev < 1 ? 1 : *h.step_dev;
        bc1 = -expm1((double)s.step * h.log1), bc2 = -expm1((double)s.step * h.log2);
    }
    s.keep = (float)(1 - lr * decay);
    s.rate = (float)(lr / bc1);
    s.root = (float)(1 / sqrt(bc2));
    s.scale = h.grad_scale ? *h.grad_scale : 1.f;
    s.skip = !isfinite(s.scale);
    s.eps = h.eps, s.b1 = h.b1, s.c1 = h.c1, s.b2 = h.b2, s.c2 = h.c2;
    return s;
}

// Root and quotient to half a step of 2^-23 (a 2^-20th of a step more, at most): the hardware's, which are right to a step, and one step of Newton's with
// the remainder, which fmaf gives exactly.  Where there is no remainder to speak of (infinities) the hardware's stays.  The compiler's forms take three
// times the instructions, which shows where a list is so small that a launch is one wave's time: 150 tensors, 1.4 M elements, 15.0 us with those, 14.7 with these,
// 14.3 with the hardware's alone; one Llama-8B layer with its norm 1282 us, 1282, 1284.
__device__ __forceinline__ float root_of(float x)
{
    const float s = __builtin_amdgcn_sqrtf(x), rest = fmaf(-s, s, x);
    return fabsf(rest) < INFINITY ? fmaf(rest, 0.5f * __builtin_amdgcn_rsqf(x), s) : s;
}
__device__ __forceinline__ float quotient(float a, float b)
{
    const float r = __builtin_amdgcn_rcpf(b), q = a * r, rest = fmaf(-q, b, a);
    return fabsf(rest) < INFINITY ? fmaf(rest, r, q) : q;
}

// One element.  No product is contracted with a sum: the new states are then the same bits as those of separate
// operations in 32 bits, and so are the codes that they are rounded to.  With 8-bit states (EIGHT) root and quotient are the hardware's, each right to a step of 2^-23
// (a move of p by 3 of them, at most, of itself): there the compiler's forms made a third of all instructions, and these bound the step; with 32-bit states memory
// does.  A v that is no normal number counts as the smallest, which the hardware's root would take for zero.
template <bool EIGHT> __device__ __forceinline__ void update(const Step& s, float g, float& p, float& m, float& v)
{
#pragma clang fp contract(off)
    g = g * s.scale;
    m = m * s.b1 + g * s.c1;
    v = v * s.b2 + g * g * s.c2;
    const float w = v < 0x1p-126f ? 0x1p-126f : v;
    if constexpr (EIGHT) p = p * s.keep - m * s.rate * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(w) * s.root + s.eps);
    else p = p * s.keep - quotient(m * s.rate, root_of(w) * s.root + s.eps);
}

template <class G, int U> __device__ __forceinline__ void zero_grads(G* g, int64_t left)
{
#pragma unroll
    for (int i = 0; i < U / 256 / 4; ++i) {
        const int c = (i * 256 + threadIdx.x) * 4;
        if (c < left) store_to<false>(g + c, left - c, Vec<G, 4>{});
    }
}

template <class G, int U, bool WHOLE>
__device__ __forceinline__ void adamw_unit(const Step& s, G* g, float* p, float* m, float* v, uint16_t* w, int64_t left, bool zero)
{
    constexpr int V = 4, N = U / 256 / V;
    Vec<G, V> xg[N];
    Vec<float, V> xp[N], xm[N], xv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        if (!WHOLE && c >= left) break;
        xg[i] = load_to<G, V, WHOLE>(g + c, left - c);
        xp[i] = load_to<float, V, WHOLE>(p + c, left - c);
        xm[i] = load_to<float, V, WHOLE>(m + c, left - c);
        xv[i] = load_to<float, V, WHOLE>(v + c, left - c);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        if (!WHOLE && c >= left) break;
#pragma unroll
        for (int e = 0; e < V; ++e) update<false>(s, to_float(xg[i].e[e]), xp[i].e[e], xm[i].e[e], xv[i].e[e]);
        store_to<WHOLE>(p + c, left - c, xp[i]);
        store_to<WHOLE>(m + c, left - c, xm[i]);
        store_to<WHOLE>(v + c, left - c, xv[i]);
        if (w) store_to<WHOLE>(w + c, left - c, rounded<V>(xp[i].e, uint16_t()));
        if (zero) store_to<WHOLE>(g + c, left - c, Vec<G, V>{});
    }
}

template <class G, int U> __global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs<Tensor32, TENSORS32> a)
{
    const int k = find(a.list.first, blockIdx.x);
    const Tensor32& t = a.list.t[k];
    const int64_t at = (int64_t)(blockIdx.x - a.list.first[k]) * U, left = t.n - at;
    const Step s = make_step(a.h, t.decay);
    G* g = static_cast<G*>(t.g) + at;
    if (s.skip) {
        if (a.h.zero) zero_grads<G, U>(g, left);
        return;
    }
    float *m = static_cast<float*>(t.m) + at, *v = static_cast<float*>(t.v) + at;
    uint16_t* w = t.w ? t.w + at : nullptr;
    if (left >= U) adamw_unit<G, U, true>(s, g, t.p + at, m, v, w, left, a.h.zero);
    else adamw_unit<G, U, false>(s, g, t.p + at, m, v, w, left, a.h.zero);
}

// ---- 8-bit states.  A block of 128 has an exponent byte E, that of its largest value rounded up to three fraction bits (at
// least 40, so that no code stands for a denormal; 255: a value was not finite, the block's values are NaN).  A code c > 0
// stands for the float of bits (E - D) 2^23 + c 2^20, c = 0 for zero: three fraction bits and the exponents from E - D to E,
// D = 15 for m (and a sign), 31 for v.
// Shifts and multiplications by turns, so that every bit of x reaches every bit of the result: the form, and the shifts 15, 13 and 16, in which
// the published hash XXH32 ends, with other odd factors.
__device__ __forceinline__ unsigned mix(unsigned x)
{
    x ^= x >> 15;
    x *= 0xB7E15163u;
    x ^= x >> 13;
    x *= 0x93C467E3u;
    return x ^ (x >> 16);
}

// `nan`: 0x7fc00000 where the block's byte is 255, else 0
template <int D> __device__ __forceinline__ float decode(unsigned code, unsigned base, unsigned nan)
{
    const unsigned mag = D == 15 ? code & 127 : code;
    const unsigned bits = mag ? base + (mag << 20) : 0;
    return __uint_as_float(bits | nan | (D == 15 ? (code & 128) << 24 : 0));
}
template <int D> __device__ __forceinline__ unsigned decode_base(unsigned exp) { return (exp - D) << 23; }
__device__ __forceinline__ unsigned decode_nan(unsigned exp) { return exp == 255 ? 0x7fc00000u : 0; }

// The largest over the 32 lanes of a block, in each of them: rotated by 8, 4, 2 and 1 of 16 lanes, then with the other 16.
__device__ __forceinline__ unsigned block_max(unsigned x)
{
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, true));
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, true));
    const auto both = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return max(both[0], both[1]);
}
__device__ __forceinline__ unsigned exponent(unsigned most)
{
    const unsigned e = (most + 0xfffffu) >> 23;
    return e >= 255 ? 255 : max(e, 40u);
}

// |x| rounded to a code, up with the probability of what is cut off (16 random bits): a step changes v by 1 - beta2 of
// itself, far less than half the distance of two codes, and rounded to nearest it would stay where it is.  What is below code
// 1 becomes 1 or 0 likewise for m, and 1 for v, by which a step divides.
// (both cases computed, one taken: a branch for each element kept them from overlapping)
__device__ __forceinline__ unsigned encode_m(float x, unsigned base, float least, unsigned random16)
{
    const unsigned bits = __float_as_uint(x) & 0x7fffffffu;
    const float size = __uint_as_float(bits);
    const unsigned low = (float)random16 * (0x1p-16f * least) < size, high = ((bits + (random16 << 4)) >> 20) - base;
    const unsigned code = __builtin_unpredictable(size >= least) ? high : low;
    return code | (__float_as_uint(x) >> 24 & 128);
}
__device__ __forceinline__ unsigned encode_v(float x, unsigned base, unsigned random16)
{
    const unsigned bits = __float_as_uint(x);
    return (unsigned)max((int)((bits + (random16 << 4)) >> 20) - (int)base, (int)min(bits, 1u));  // (v is not negative)
}

// Four elements of a lane at a time, so that every access of a wave is contiguous (with eight, the two halves of a lane's p
// and g are 32 bytes from the next lane's).
template <class G, int U, bool WHOLE>
__device__ __forceinline__ void adamw8_unit(const Step& s, G* g, float* p, uint8_t* m, uint8_t* v, uint8_t* me, uint8_t* ve, uint16_t* w, unsigned at,
                                            unsigned key, int64_t left, bool zero)
{
    constexpr int V = 4, N = U / 256 / V;
    Vec<G, V> xg[N];
    Vec<float, V> xp[N];
    Vec<uint8_t, V> xm[N], xv[N];
    unsigned em[N], ev[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        if (WHOLE || c < left) {
            xg[i] = load_to<G, V, WHOLE>(g + c, left - c);
            xp[i] = load_to<float, V, WHOLE>(p + c, left - c);
            xm[i] = load_to<uint8_t, V, WHOLE>(m + c, left - c);
            xv[i] = load_to<uint8_t, V, WHOLE>(v + c, left - c);
            em[i] = me[c / BLOCK], ev[i] = ve[c / BLOCK];
        } else {  // no element: zeros, which do not count in the block's largest
            xg[i] = {}, xp[i] = {}, xm[i] = {}, xv[i] = {}, em[i] = ev[i] = 0;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        float fm[V], fv[V];
        unsigned most_m = 0, most_v = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            fm[e] = decode<15>(xm[i].e[e], decode_base<15>(em[i]), decode_nan(em[i]));
            fv[e] = decode<31>(xv[i].e[e], decode_base<31>(ev[i]), decode_nan(ev[i]));
            update<true>(s, to_float(xg[i].e[e]), xp[i].e[e], fm[e], fv[e]);
            if (WHOLE || c + e < left) {  // (a NaN of the block's exponent must not come from behind the end)
                most_m = max(most_m, __float_as_uint(fm[e]) & 0x7fffffffu);
                most_v = max(most_v, __float_as_uint(fv[e]) & 0x7fffffffu);
            }
        }
        const unsigned nm = exponent(block_max(most_m)), nv = exponent(block_max(most_v));
        if (!WHOLE && c >= left) continue;
        const unsigned base_m = (nm - 15) << 3, base_v = (nv - 31) << 3;
        const float least = __uint_as_float((base_m + 1) << 20);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const unsigned random = mix((at + c + e) * 0x9E3779B1u ^ key);
            xm[i].e[e] = (uint8_t)encode_m(fm[e], base_m, least, random & 0xffff);
            xv[i].e[e] = (uint8_t)encode_v(fv[e], base_v, random >> 16);
        }
        if (nm == 255) xm[i] = {};
        if (nv == 255) xv[i] = {};
        store_to<WHOLE>(m + c, left - c, xm[i]);
        store_to<WHOLE>(v + c, left - c, xv[i]);
        if (c % BLOCK == 0) me[c / BLOCK] = (uint8_t)nm, ve[c / BLOCK] = (uint8_t)nv;
        store_to<WHOLE>(p + c, left - c, xp[i]);
        if (zero) store_to<WHOLE>(g + c, left - c, Vec<G, V>{});
        if (w) store_to<WHOLE>(w + c, left - c, rounded<V>(xp[i].e, uint16_t()));
    }
}

template <class G, int U> __global__ __launch_bounds__(256) void adamw8_kernel(AdamwArgs<Tensor8, TENSORS8> a)
{
    const int k = find(a.list.first, blockIdx.x);
    const Tensor8& t = a.list.t[k];
    const int64_t at = (int64_t)(blockIdx.x - a.list.first[k]) * U, left = t.n - at;
    const Step s = make_step(a.h, t.decay);
    G* g = static_cast<G*>(t.g) + at;
    if (s.skip) {
        if (a.h.zero) zero_grads<G, U>(g, left);
        return;
    }
    unsigned key = mix(mix(mix(a.h.seed ^ 0x243F6A88u) ^ (unsigned)s.step * 0x9E3779B1u) ^ t.ordinal * 0x85A308D3u);
    if (at >> 32) key = mix(key + (unsigned)(at >> 32));
    uint8_t *m = static_cast<uint8_t*>(t.m) + at, *v = static_cast<uint8_t*>(t.v) + at, *me = t.m_exp + at / BLOCK, *ve = t.v_exp + at / BLOCK;
    uint16_t* w = t.w ? t.w + at : nullptr;
    if (left >= U) adamw8_unit<G, U, true>(s, g, t.p + at, m, v, me, ve, w, (unsigned)at, key, left, a.h.zero);
    else adamw8_unit<G, U, false>(s, g, t.p + at, m, v, me, ve, w, (unsigned)at, key, left, a.h.zero);
}

struct Unpacked {
    const uint8_t *m, *v, *m_exp, *v_exp;
    uint16_t *m_value, *v_value;
    int64_t n;
};
constexpr int TENSORS_UNPACK = 64;
struct UnpackArgs {
    List<Unpacked, TENSORS_UNPACK> list;
};

// Four significant bits: bfloat16 holds them, in the upper half of the float's bits.
template <bool WHOLE> __device__ __forceinline__ void unpack_unit(const Unpacked& t, int64_t at, int64_t left)
{
    constexpr int V = 8, N = UNIT / 256 / V;
    Vec<uint8_t, V> m[N], v[N];
    unsigned em[N], ev[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        if (!WHOLE && c >= left) break;
        m[i] = load_to<uint8_t, V, WHOLE>(t.m + at + c, left - c), v[i] = load_to<uint8_t, V, WHOLE>(t.v + at + c, left - c);
        em[i] = t.m_exp[(at + c) / BLOCK], ev[i] = t.v_exp[(at + c) / BLOCK];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = (i * 256 + threadIdx.x) * V;
        if (!WHOLE && c >= left) break;
        Vec<uint16_t, V> ym, yv;
#pragma unroll
        for (int e = 0; e < V; ++e)
            ym.e[e] = (uint16_t)(__float_as_uint(decode<15>(m[i].e[e], decode_base<15>(em[i]), decode_nan(em[i]))) >> 16),
            yv.e[e] = (uint16_t)(__float_as_uint(decode<31>(v[i].e[e], decode_base<31>(ev[i]), decode_nan(ev[i]))) >> 16);
        store_to<WHOLE>(t.m_value + at + c, left - c, ym);
        store_to<WHOLE>(t.v_value + at + c, left - c, yv);
    }
}

__global__ __launch_bounds__(256) void adamw_unpack_kernel(UnpackArgs a)
{
    const int k = find(a.list.first, blockIdx.x);
    const Unpacked& t = a.list.t[k];
    const int64_t at = (int64_t)(blockIdx.x - a.list.first[k]) * UNIT, left = t.n - at;
    if (left >= UNIT) unpack_unit<true>(t, at, left);
    else unpack_unit<false>(t, at, left);
}

// ---- host
// Cuts `count` tensors into launches: at most N of them and MOST_UNITS units each.  take(k) fills the list's next entry,
// launch(units) sends the list off.
template <class L, int N, class Take, class Launch> int in_launches(const fpdt_tw_param* params, int count, int unit, L& list, Take take, Launch launch)
{
    int used = 0;
    unsigned units = 0;
    auto send = [&]() {
        if (!used) return;
        for (int i = used; i < N; ++i) list.first[i] = ~0u;
        launch(units);
        used = 0, units = 0;
    };
    for (int k = 0; k < count; ++k) {
        if (params[k].n == 0) continue;
        const unsigned need = (unsigned)((params[k].n + unit - 1) / unit);
        if (used == N || units + need > MOST_UNITS) send();
        list.first[used] = units;
        take(list.t[used], k);
        units += need;
        ++used;
    }
    send();
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

// Units of a list, in all
int64_t units_of(const fpdt_tw_param* params, int count, int unit)
{
    int64_t n = 0;
    for (int k = 0; k < count; ++k) n += (params[k].n + unit - 1) / unit;
    return n;
}

int check_list(const fpdt_tw_param* params, int count, int grad_dtype)
{
    if (!params || count <= 0) return fail(TW_INVALID, "params NULL or count not positive");
    if (grad_dtype != FPDT_TW_F32 && grad_dtype != FPDT_TW_BF16) return fail(TW_INVALID, "unknown grad_dtype %d", grad_dtype);
    for (int k = 0; k < count; ++k) {
        if (params[k].n < 0) return fail(TW_INVALID, "tensor %d has %lld elements", k, (long long)params[k].n);
        if (params[k].n > MOST_ELEMENTS) return fail(TW_UNSUPPORTED, "tensor %d: %lld elements are beyond the launch limits", k, (long long)params[k].n);
        if (params[k].n && (!params[k].g || misaligned(params[k].g, grad_dtype == FPDT_TW_F32 ? 4 : 2)))
            return fail(TW_INVALID, "tensor %d: g is NULL or not aligned to its elements", k);
    }
    return TW_OK;
}

}  // namespace

extern "C" {

size_t fpdt_tw_grad_norm_workspace_bytes(int count)
{
    if (count <= 0) return 0;
    return ((size_t)count + NORM_TENSORS - 1) / NORM_TENSORS * NORM_GROUPS * sizeof(double);
}

int fpdt_tw_grad_norm(const fpdt_tw_param* params, int count, int grad_dtype, double max_norm, float* out, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    int rc = check_list(params, count, grad_dtype);
    if (rc != TW_OK) return rc;
    if (!out || misaligned(out, 4)) return fail(TW_INVALID, "out is NULL or not aligned to its elements");
    if (!(max_norm > 0)) return fail(TW_INVALID, "max_norm must be positive");
    // (a list needs one launch for each NORM_TENSORS tensors then)
    const int64_t all = units_of(params, count, NORM_UNIT);
    const int unit = all >= ENOUGH ? NORM_UNIT : SMALL_NORM_UNIT;
    if (all > MOST_UNITS) return fail(TW_UNSUPPORTED, "the list's elements are beyond the launch limits");
    const size_t need = fpdt_tw_grad_norm_workspace_bytes(count);
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256))
        return fail(TW_WORKSPACE, "workspace NULL, misaligned or too small (%zu < %zu bytes)", workspace_bytes, need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    NormArgs a;
    double* partial = static_cast<double*>(workspace);
    int n = 0;
    rc = in_launches<decltype(a.list), NORM_TENSORS>(
        params, count, unit, a.list, [&](NormTensor& t, int k) { t = {params[k].g, params[k].n}; },
        [&](unsigned units) {
            const unsigned grid = units < NORM_GROUPS ? units : NORM_GROUPS;
            a.partial = partial + n, a.units = units;
            n += (int)grid;
            const bool wide = grad_dtype == FPDT_TW_F32;
            if (unit == NORM_UNIT && wide) grad_norm_kernel<float, NORM_UNIT><<<grid, 256, 0, st>>>(a);
            else if (unit == NORM_UNIT) grad_norm_kernel<uint16_t, NORM_UNIT><<<grid, 256, 0, st>>>(a);
            else if (wide) grad_norm_kernel<float, SMALL_NORM_UNIT><<<grid, 256, 0, st>>>(a);
            else grad_norm_kernel<uint16_t, SMALL_NORM_UNIT><<<grid, 256, 0, st>>>(a);
        });
    if (rc != TW_OK) return rc;
    grad_norm_end_kernel<<<1, 1024, 0, st>>>(partial, n, max_norm, out);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

int fpdt_tw_adamw_step(const fpdt_tw_param* params, int count, int grad_dtype, int state_bits, double lr, double beta1, double beta2, double eps, int64_t step,
                       const float* lr_dev, const int64_t* step_dev, const float* grad_scale, unsigned seed, unsigned flags, void* stream)
{
    clear_error();
    int rc = check_list(params, count, grad_dtype);
    if (rc != TW_OK) return rc;
    if (state_bits != 32 && state_bits != 8) return fail(TW_INVALID, "state_bits=%d must be 32 or 8", state_bits);
    if (!lr_dev && !(std::isfinite(lr) && lr >= 0)) return fail(TW_INVALID, "lr must be finite and not negative");
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1)) return fail(TW_INVALID, "beta1 and beta2 must be in [0, 1)");
    if (!(std::isfinite(eps) && eps >= 0)) return fail(TW_INVALID, "eps must be finite and not negative");
    if (!step_dev && step < 1) return fail(TW_INVALID, "step counts from 1");
    if (misaligned(lr_dev, 4) || misaligned(step_dev, 8) || misaligned(grad_scale, 4)) return fail(TW_INVALID, "lr_dev, step_dev or grad_scale is not aligned");
    if (flags & ~(unsigned)FPDT_TW_ADAMW_ZERO_GRAD) return fail(TW_INVALID, "unknown flag bits 0x%x", flags);
    const size_t state = state_bits == 32 ? 4 : 1;
    for (int k = 0; k < count; ++k) {
        const fpdt_tw_param& t = params[k];
        if (!t.n) continue;
        if (!t.p || !t.m || !t.v || (state_bits == 8 && (!t.m_exp || !t.v_exp))) return fail(TW_INVALID, "tensor %d: NULL pointer", k);
        if (misaligned(t.p, 4) || misaligned(t.w, 2) || misaligned(t.m, state) || misaligned(t.v, state))
            return fail(TW_INVALID, "tensor %d: a pointer is not aligned to its elements", k);
        if (!std::isfinite(t.weight_decay)) return fail(TW_INVALID, "tensor %d: weight_decay must be finite", k);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    AdamwHyper h;
    h.lr = lr, h.log1 = std::log(beta1), h.log2 = std::log(beta2);
    h.bc1 = -std::expm1((double)step * h.log1), h.bc2 = -std::expm1((double)step * h.log2);
    h.lr_dev = lr_dev, h.step_dev = step_dev, h.grad_scale = grad_scale, h.step = step;
    h.b1 = (float)beta1, h.c1 = (float)(1 - beta1), h.b2 = (float)beta2, h.c2 = (float)(1 - beta2), h.eps = (float)eps;
    h.seed = seed, h.zero = (flags & FPDT_TW_ADAMW_ZERO_GRAD) != 0;
    auto common = [&](Tensor32& t, int k) {
        const fpdt_tw_param& x = params[k];
        t.p = x.p, t.w = static_cast<uint16_t*>(x.w), t.g = x.g, t.m = x.m, t.v = x.v, t.n = x.n, t.decay = x.weight_decay;
    };
    const int large = state_bits == 32 ? UNIT : UNIT8, unit = units_of(params, count, large) >= ENOUGH ? large : SMALL_UNIT;
    const bool wide = grad_dtype == FPDT_TW_F32;
    if (state_bits == 32) {
        AdamwArgs<Tensor32, TENSORS32> a;
        a.h = h;
        return in_launches<decltype(a.list), TENSORS32>(params, count, unit, a.list, common, [&](unsigned units) {
            if (unit == UNIT && wide) adamw_kernel<float, UNIT><<<units, 256, 0, st>>>(a);
            else if (unit == UNIT) adamw_kernel<uint16_t, UNIT><<<units, 256, 0, st>>>(a);
            else if (wide) adamw_kernel<float, SMALL_UNIT><<<units, 256, 0, st>>>(a);
            else adamw_kernel<uint16_t, SMALL_UNIT><<<units, 256, 0, st>>>(a);
        });
    }
    AdamwArgs<Tensor8, TENSORS8> a;
    a.h = h;
    return in_launches<decltype(a.list), TENSORS8>(
        params, count, unit, a.list,
        [&](Tensor8& t, int k) {
            common(t, k);
            t.m_exp = params[k].m_exp, t.v_exp = params[k].v_exp, t.ordinal = (unsigned)k, t.pad = 0;
        },
        [&](unsigned units) {
            if (unit == UNIT8 && wide) adamw8_kernel<float, UNIT8><<<units, 256, 0, st>>>(a);
            else if (unit == UNIT8) adamw8_kernel<uint16_t, UNIT8><<<units, 256, 0, st>>>(a);
            else if (wide) adamw8_kernel<float, SMALL_UNIT><<<units, 256, 0, st>>>(a);
            else adamw8_kernel<uint16_t, SMALL_UNIT><<<units, 256, 0, st>>>(a);
        });
}

int fpdt_tw_adamw_unpack(const fpdt_tw_param* params, int count, void* stream)
{
    clear_error();
    if (!params || count <= 0) return fail(TW_INVALID, "params NULL or count not positive");
    for (int k = 0; k < count; ++k) {
        const fpdt_tw_param& t = params[k];
        if (t.n < 0) return fail(TW_INVALID, "tensor %d has %lld elements", k, (long long)t.n);
        if (t.n > MOST_ELEMENTS) return fail(TW_UNSUPPORTED, "tensor %d: %lld elements are beyond the launch limits", k, (long long)t.n);
        if (t.n && (!t.m || !t.v || !t.m_exp || !t.v_exp || !t.m_value || !t.v_value)) return fail(TW_INVALID, "tensor %d: NULL pointer", k);
        if (misaligned(t.m_value, 2) || misaligned(t.v_value, 2)) return fail(TW_INVALID, "tensor %d: a pointer is not aligned to its elements", k);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    UnpackArgs a;
    return in_launches<decltype(a.list), TENSORS_UNPACK>(
        params, count, UNIT, a.list,
        [&](Unpacked& t, int k) {
            const fpdt_tw_param& x = params[k];
            t = {static_cast<const uint8_t*>(x.m), static_cast<const uint8_t*>(x.v), x.m_exp, x.v_exp, static_cast<uint16_t*>(x.m_value),
                 static_cast<uint16_t*>(x.v_value), x.n};
        },
        [&](unsigned units) { adamw_unpack_kernel<<<units, 256, 0, st>>>(a); });
}

}  // extern "C"
