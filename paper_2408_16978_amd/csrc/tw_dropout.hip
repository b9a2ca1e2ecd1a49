// Dropout with the residual add (include/fpdt_tokenwise.h: fpdt_tw_dropout_*).
//
//     y = keep x s + r,   keep by 16 bits of a counter-based generator for each element
//
// Bound by the memory: the generator's ten rounds of two 32 x 32 -> 64 bit products serve eight elements, and run under the accesses (65536 x 2560 in bf16 with
// the residual: 157-159 us between events around many calls, 6.3-6.4 TB/s; 162-168 in a kernel trace; vector instructions in half of the time).  Sixteen bits an element and not 32, which would take twice the rounds: p is a multiple of 2^-16,
// and the scale that of the share that is kept.
#include <cmath>

#include "../../include/fpdt_tokenwise.h"
#include "tw_common.h"

namespace {

using namespace fpdt_tw;

// Philox4x32-10 as it was published (Salmon et al. 2011): its two multipliers, and the two Weyl increments of the key.
__device__ __forceinline__ uintx4 philox(uintx4 c, unsigned k0, unsigned k1)
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        c = uintx4{(unsigned)(b >> 32) ^ c[1] ^ k0, (unsigned)b, (unsigned)(a >> 32) ^ c[3] ^ k1, (unsigned)a};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

constexpr int V = 8;  // elements of a counter
// Eight elements in accesses of 16 bytes
template <class T> __device__ __forceinline__ Vec<T, V> load8(const T* p)
{
    constexpr int A = 16 / sizeof(T);
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; i += A) {
        const Vec<T, A> a = load_once<A>(p + i);
#pragma unroll
        for (int e = 0; e < A; ++e) v.e[i + e] = a.e[e];
    }
    return v;
}
template <class T> __device__ __forceinline__ void store8(T* p, const Vec<T, V>& v)
{
    constexpr int A = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < V; i += A) {
        Vec<T, A> a;
#pragma unroll
        for (int e = 0; e < A; ++e) a.e[e] = v.e[i + e];
        store_once(p + i, a);
    }
}

// A thread takes the elements of a counter: number `first` need not begin one, the last need not end one.
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* X, const T* R, T* Y, int64_t n, int64_t first, unsigned dropped, float scale, uint64_t seed, int64_t step,
                                                      const int64_t* step_dev)
{
    if (step_dev) step = *step_dev;
    const int64_t from = first / V, blocks = (first + n - 1) / V - from + 1;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < blocks; i += (int64_t)gridDim.x * 256) {
        const int64_t b = from + i, at = b * V - first;  // the counter's first element within the call (below 0: it is not of the call)
        const bool whole = at >= 0 && at + V <= n;
        Vec<T, V> x = {}, r = {};
        if (whole) {
            x = load8(X + at);
            if (R) r = load8(R + at);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at + e >= 0 && at + e < n) {
                    x.e[e] = X[at + e];
                    if (R) r.e[e] = R[at + e];
                }
        }
        const uintx4 bits = philox(uintx4{(unsigned)b, (unsigned)(b >> 32), (unsigned)step, (unsigned)(step >> 32)}, (unsigned)seed, (unsigned)(seed >> 32));
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const unsigned mine = e % 2 ? bits[e / 2] >> 16 : bits[e / 2] & 0xffffu;
            y[e] = mine >= dropped ? to_float(x.e[e]) * scale : 0.f;
            if (R) y[e] += to_float(r.e[e]);
        }
        const Vec<T, V> out = rounded<V>(y, T());
        if (whole) {
            store8(Y + at, out);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at + e >= 0 && at + e < n) Y[at + e] = out.e[e];
        }
    }
}

int dropout(const void* X, const void* R, void* Y, int64_t n, int64_t first, double p, uint64_t seed, int64_t step, const int64_t* step_dev, int dtype, void* stream)
{
    clear_error();
    if (!X || !Y) return fail(TW_INVALID, "NULL tensor pointer");
    if (n <= 0 || first < 0) return fail(TW_INVALID, "n must be positive, and first not negative");
    if (!(p >= 0 && p <= 1)) return fail(TW_INVALID, "p must be in [0, 1]");
    if (dtype != FPDT_TW_F32 && dtype != FPDT_TW_BF16) return fail(TW_INVALID, "unknown dtype %d", dtype);
    if (n >= (int64_t)1 << 61 || first >= ((int64_t)1 << 62) - n) return fail(TW_UNSUPPORTED, "first + n beyond 2^62");
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, bytes = (size_t)n * size;
    if (misaligned(X, size) || misaligned(R, size) || misaligned(Y, size) || misaligned(step_dev, 8)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    for (const void* in : {X, R})
        if (in && in != Y && ranges_meet(in, bytes, Y, bytes)) return fail(TW_INVALID, "the output overlaps an input without being it");
    if (step_dev && ranges_meet(step_dev, 8, Y, bytes)) return fail(TW_INVALID, "the output overlaps step_dev");
    const unsigned dropped = (unsigned)std::nearbyint(p * 65536.);
    const float scale = dropped < 65536 ? (float)(65536. / (65536. - dropped)) : 0.f;
    const int64_t blocks = (n + 2 * V - 2) / V, groups = (blocks + 255) / 256;
    const unsigned grid = (unsigned)(groups < 1 << 20 ? groups : 1 << 20);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (size == 4)
        dropout_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float*>(X), static_cast<const float*>(R), static_cast<float*>(Y), n, first, dropped, scale, seed, step, step_dev);
    else
        dropout_kernel<uint16_t>
            <<<grid, 256, 0, st>>>(static_cast<const uint16_t*>(X), static_cast<const uint16_t*>(R), static_cast<uint16_t*>(Y), n, first, dropped, scale, seed, step, step_dev);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // namespace

extern "C" {

int fpdt_tw_dropout_fwd(const void* X, const void* R, void* Y, int64_t n, int64_t first, double p, uint64_t seed, int64_t step, const int64_t* step_dev, int dtype,
                        void* stream)
{
    return dropout(X, R, Y, n, first, p, seed, step, step_dev, dtype, stream);
}

int fpdt_tw_dropout_bwd(const void* dY, void* dX, int64_t n, int64_t first, double p, uint64_t seed, int64_t step, const int64_t* step_dev, int dtype, void* stream)
{
    return dropout(dY, nullptr, dX, n, first, p, seed, step, step_dev, dtype, stream);
}

}  // extern "C"
