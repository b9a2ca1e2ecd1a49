// What the sources of the token-wise library share: status codes and the error text (tokenwise.hip), accesses of
// several elements, conversions, sums over lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fpdt_tw {

enum { TW_OK = 0, TW_INVALID = 1, TW_UNSUPPORTED = 2, TW_WORKSPACE = 3, TW_HIP = 4 };

// Sets the calling thread's error text and returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

#define HIP_TRY(expr)                                                                            \
    do {                                                                                         \
        hipError_t e_ = (expr);                                                                  \
        if (e_ != hipSuccess) return fail(TW_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

// Do the byte ranges [a, a + na) and [b, b + nb) meet?
inline bool ranges_meet(const void* a, size_t na, const void* b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
}

inline bool misaligned(const void* p, size_t by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }

// V elements in one access.  The address need only be aligned to an element: global memory is read and written at
// any address here, at the price of the cache lines that an access touches.
template <class T, int V> struct Vec {
    T e[V];
};
template <int BYTES, int ALIGN> struct Raw;
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
#define FPDT_TW_RAW(BYTES, ALIGN, TYPE)                                \
    template <> struct Raw<BYTES, ALIGN> {                             \
        typedef TYPE type __attribute__((aligned(ALIGN), may_alias));  \
    };
FPDT_TW_RAW(4, 1, unsigned)
FPDT_TW_RAW(8, 1, uintx2)
FPDT_TW_RAW(2, 2, uint16_t)
FPDT_TW_RAW(4, 2, unsigned)
FPDT_TW_RAW(8, 2, uintx2)
FPDT_TW_RAW(16, 2, uintx4)
FPDT_TW_RAW(4, 4, unsigned)
FPDT_TW_RAW(8, 4, uintx2)
FPDT_TW_RAW(16, 4, uintx4)
#undef FPDT_TW_RAW
template <int V, class T> __device__ __forceinline__ Vec<T, V> load(const T* p)
{
    typedef typename Raw<sizeof(T) * V, sizeof(T)>::type R;
    return __builtin_bit_cast(Vec<T, V>, *reinterpret_cast<const R*>(p));
}
template <int V, class T> __device__ __forceinline__ void store(T* p, const Vec<T, V>& v)
{
    typedef typename Raw<sizeof(T) * V, sizeof(T)>::type R;
    *reinterpret_cast<R*>(p) = __builtin_bit_cast(R, v);
}
// The same past the caches, for what passes through once.  2 GiB read 7.1 TB/s (6.3 without), copied 6.5 (6.1), with 4
// tensors read and 3 of them written 5.8 (5.4).
template <int V, class T> __device__ __forceinline__ Vec<T, V> load_once(const T* p)
{
    typedef typename Raw<sizeof(T) * V, sizeof(T)>::type R;
    return __builtin_bit_cast(Vec<T, V>, __builtin_nontemporal_load(reinterpret_cast<const R*>(p)));
}
template <int V, class T> __device__ __forceinline__ void store_once(T* p, const Vec<T, V>& v)
{
    typedef typename Raw<sizeof(T) * V, sizeof(T)>::type R;
    __builtin_nontemporal_store(__builtin_bit_cast(R, v), reinterpret_cast<R*>(p));
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
// rounded to the type, to nearest even
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

template <int V> __device__ __forceinline__ Vec<float, V> rounded(const float* x, float)
{
    Vec<float, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = x[i];
    return v;
}
template <int V> __device__ __forceinline__ Vec<uint16_t, V> rounded(const float* x, uint16_t)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    Vec<uint16_t, V> v;
    if constexpr (V == 1) {
        v.e[0] = from_float<uint16_t>(x[0]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const unsigned two = __builtin_bit_cast(unsigned, __builtin_convertvector((floatx2{x[i], x[i + 1]}), bf16x2));
            v.e[i] = (uint16_t)two;
            v.e[i + 1] = (uint16_t)(two >> 16);
        }
    }
    return v;
}

template <int N> struct Int {
    static constexpr int value = N;
};

// Sum over LANES consecutive lanes (16, 32 or 64, from a multiple of them on), in every one of them: rotations by 8, 4, 2 and 1 of 16
// lanes, then with the other rows of 16.  All lanes of the rows have to be active.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(LANES == 16 || LANES == 32 || LANES == 64, "");
    auto turned = [](float x, auto by) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x120 + decltype(by)::value, 0xf, 0xf, true)); };
    v += turned(v, Int<8>());
    v += turned(v, Int<4>());
    v += turned(v, Int<2>());
    v += turned(v, Int<1>());
    if constexpr (LANES >= 32) {
        const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    if constexpr (LANES == 64) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    }
    return v;
}
__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}

}  // namespace fpdt_tw
