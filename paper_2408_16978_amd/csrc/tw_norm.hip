// Normalisation of rows with the residual add in front of it (include/fpdt_tokenwise.h: fpdt_tw_norm_*).
//
//     s = x + r,   u = (s - mean) rstd,   y = u w + b          (RMS: mean = 0, b = 0)
//     h = dy w,    dx = rstd (h - mean(h) - u mean(h u)) + dr  (RMS: without mean(h))
//     dw += sum_rows dy u,   db += sum_rows dy
//
// Bound by the memory: a row stays in the registers of the lanes that read it, so each tensor is read or written once.
#include <cmath>
#include <type_traits>

#include "../../include/fpdt_tokenwise.h"
#include "tw_common.h"

namespace {

using namespace fpdt_tw;

constexpr int MOST_HIDDEN = 16384;

// A row belongs to LANES = 16, 32 or 64 lanes of a wave, in workgroups of 256 threads, or (LANES = 0) to all threads of a
// workgroup, any number of waves up to 16, so that few of them are idle whatever the width.
constexpr int SMALL = 256;
template <int LANES> __device__ __forceinline__ int row_lanes() { return LANES ? LANES : (int)blockDim.x; }
template <int LANES> __device__ __forceinline__ int row_lane() { return LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x; }
template <int LANES> __device__ __forceinline__ int row_of() { return LANES ? threadIdx.x / (LANES ? LANES : 1) : 0; }

// Sums of N values over the threads of a row, in every one of them.  `red` holds the sums of 16 waves, twice and used by
// turns, so that one barrier is enough.
template <int LANES, int N> struct RowSum {
    float (*red)[N][16];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = lanes_sum<LANES ? LANES : 64>(v[n]);
        if constexpr (LANES == 0) {
            const int waves = blockDim.x / 64;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int n = 0; n < N; ++n) red[turn][n][threadIdx.x / 64] = v[n];
            __syncthreads();
            const int w = threadIdx.x & 15;
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] = lanes_sum<16>(w < waves ? red[turn][n][w] : 0.f);
            turn ^= 1;
        }
    }
};

// Access i of a lane covers columns [c, c + V), c = (i lanes + lane) V.  WHOLE: hidden is a multiple of V; if not, the last
// access of a row is cut off.  Past the caches in either case, also where rows end within a cache line (through them, 1000
// columns took 229 us for 198, 1001 280 for 241).
template <bool WHOLE, int V, class T> __device__ __forceinline__ Vec<T, V> load_cut(const T* p, int c, int hidden)
{
    if (WHOLE || c + V <= hidden) return load_once<V>(p + c);
    Vec<T, V> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = c + e < hidden ? p[c + e] : T(0);
    return v;
}
template <bool WHOLE, int V, class T> __device__ __forceinline__ void store_cut(T* p, int c, int hidden, const Vec<T, V>& v)
{
    if (WHOLE || c + V <= hidden) {
        store_once(p + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < hidden) p[c + e] = v.e[e];
    }
}
// What all rows share: kept by the caches.
template <bool WHOLE, int V, class T> __device__ __forceinline__ Vec<T, V> load_row(const T* p, int c, int hidden)
{
    if (WHOLE || c + V <= hidden) return load<V>(p + c);
    return load_cut<WHOLE, V>(p, c, hidden);
}

// What was made of v so far is not kept: it is made again from v, which for bf16 takes half the registers.
template <class T, int V> __device__ __forceinline__ void forget(Vec<T, V>& v)
{
    unsigned x[sizeof v / 4];
    __builtin_memcpy(x, &v, sizeof v);
#pragma unroll
    for (unsigned& word : x) asm volatile("" : "+v"(word));
    __builtin_memcpy(&v, x, sizeof v);
}

// A sum over a row, divided by its length: rounded once, which a product with a 1 / hidden in fp32 is not (a constant row of 1000 then kept a deviation of 6e-5,
// 2% of what eps = 1e-5 stands for).  inv is 1 / hidden, an argument of the kernel that costs no vector registers.
__device__ __forceinline__ float mean_of(float sum, double inv) { return (float)(sum * inv); }

// 1 / sqrt(sum inv + eps), rounded once: the hardware's root to a step of 2^-23 and one step of Newton's in 64 bits (a root and a quotient in fp32 are
// two roundings).  What the hardware takes for zero, and infinities, go through fp32's own.
__device__ __forceinline__ float rstd_of(float sum, double inv, float eps)
{
    const double q = fma((double)sum, inv, (double)eps);
    const float f = (float)q;
    if (!(f >= 0x1p-126f && f < INFINITY)) return 1.f / sqrtf(f);
    const double r = __builtin_amdgcn_rsqf(f);
    return (float)fma(0.5 * r, fma(-r * r, q, 1.), r);
}

// Rows of NA accesses of V elements a lane.
template <class T, int LANES, int NA, bool LAYER, bool WHOLE>
__global__ __launch_bounds__((LANES ? SMALL : 1024)) void norm_fwd_kernel(const T* X, const T* R, const T* W, const T* B, T* S, T* Y, float* stats, int64_t rows,
                                                                          int hidden, double inv, float eps)
{
    constexpr int V = 16 / sizeof(T), ROWS = LANES ? SMALL / (LANES ? LANES : 1) : 1;
    __shared__ float red[2][1][16];
    RowSum<LANES, 1> sum{red};
    const int lanes = row_lanes<LANES>(), lane = row_lane<LANES>();
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + row_of<LANES>(), at = row * hidden;
        const int width = row < rows ? hidden : 0;  // (lanes without a row take part in the sums)
        Vec<T, V> x[NA], r[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            x[i] = {};
            if (c < width) x[i] = load_cut<WHOLE, V>(X + at, c, hidden);
        }
        if (R) {
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                const int c = (i * lanes + lane) * V;
                if (c < width) r[i] = load_cut<WHOLE, V>(R + at, c, hidden);
            }
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                const int c = (i * lanes + lane) * V;
                if (c >= width) continue;
                float s[V];
#pragma unroll
                for (int e = 0; e < V; ++e) s[e] = to_float(x[i].e[e]) + to_float(r[i].e[e]);
                x[i] = rounded<V>(s, T());  // what the backward reads is what is normalised
                if (S) store_cut<WHOLE, V>(S + at, c, hidden, x[i]);
            }
        }
        float mean = 0.f;
        if (LAYER) {
            float v[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) v[0] += to_float(x[i].e[e]);
            sum(v);
            mean = mean_of(v[0], inv);
        }
        float v[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            if (LAYER && WHOLE && c >= width) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = LAYER && !WHOLE && c + e >= width ? 0.f : to_float(x[i].e[e]) - mean;
                v[0] = fmaf(d, d, v[0]);
            }
        }
        sum(v);
        const float rstd = rstd_of(v[0], inv, eps);
        if (stats && lane == 0 && width) {
            if (LAYER) stats[row] = mean;
            stats[(LAYER ? rows : 0) + row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            if (c >= width) continue;
            forget(x[i]);
            float y[V];
            const Vec<T, V> w = load_row<WHOLE, V>(W, c, hidden);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = (to_float(x[i].e[e]) - mean) * rstd * to_float(w.e[e]);
            if (LAYER && B) {
                const Vec<T, V> b = load_row<WHOLE, V>(B, c, hidden);
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] += to_float(b.e[e]);
            }
            store_cut<WHOLE, V>(Y + at, c, hidden, rounded<V>(y, T()));
        }
    }
}

// Waves on a SIMD that the backward's registers are held to, and workgroups on the whole chip by that: one more than fit at
// once would walk its rows when the others are done.  64K x 4096 in bf16 (8 waves a row): 768 workgroups 373 us, 1024 of them 439, 1536 378.
constexpr int bwd_waves(int accesses) { return accesses == 1 ? 6 : 4; }
// Each leaves a row of partial sums for dw and one for db, which are read again: 16 MB a sum at most (512 rows of 8192 columns, 256 of 16384).
constexpr int bwd_groups(int threads, int accesses, int hidden)
{
    const int n = 256 * (bwd_waves(accesses) * 4 / (threads / 64)), most = hidden <= 2048 ? 2048 : 1024;
    return n < most ? n : most;
}

// Groups of LANES threads walk the rows; a thread keeps its columns' shares of dw and db in registers, a workgroup's
// groups add theirs up in LDS and leave one row of partial sums each for norm_sums_kernel: no atomics, the same order
// of sums in every call.
template <class T, int LANES, int NA, bool LAYER, bool WHOLE>
__global__ __launch_bounds__((LANES ? SMALL : 1024), bwd_waves(NA)) void norm_bwd_kernel(const T* S, const T* W, const float* stats, const T* dY, const T* dR, T* dX,
                                                                                         float* partial, int64_t rows, int hidden, double inv, bool want_w, bool want_b)
{
    constexpr int V = 16 / sizeof(T), ROWS = LANES ? SMALL / (LANES ? LANES : 1) : 1, N = LAYER ? 2 : 1;
    __shared__ float red[2][N][16];
    __shared__ float lds[LANES ? NA * V * SMALL : 1];
    RowSum<LANES, N> sum{red};
    const int lanes = row_lanes<LANES>(), lane = row_lane<LANES>();
    Vec<T, V> w[NA];
    float dw[NA][V], db[NA][V];
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int c = (i * lanes + lane) * V;
        w[i] = {};
        if (c < hidden) w[i] = load_row<WHOLE, V>(W, c, hidden);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[i][e] = db[i][e] = 0.f;
    }
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < rows; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + row_of<LANES>(), at = row * hidden;
        const int width = row < rows ? hidden : 0;  // (lanes without a row take part in the sums, with zeros)
        Vec<T, V> x[NA], y[NA], r[NA];
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            x[i] = {}, y[i] = {};
            if (c < width) x[i] = load_cut<WHOLE, V>(S + at, c, hidden), y[i] = load_cut<WHOLE, V>(dY + at, c, hidden);
        }
        if (dR)
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                const int c = (i * lanes + lane) * V;
                if (c < width) r[i] = load_cut<WHOLE, V>(dR + at, c, hidden);
            }
        const float mean = LAYER && width ? stats[row] : 0.f, rstd = width ? stats[(LAYER ? rows : 0) + row] : 0.f;
        float v[N] = {};
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            if (c >= width) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (!WHOLE && c + e >= hidden) continue;
                const float dy = to_float(y[i].e[e]);
                const float u = (to_float(x[i].e[e]) - mean) * rstd, h = dy * to_float(w[i].e[e]);
                v[0] = fmaf(h, u, v[0]);
                if (LAYER) v[N - 1] += h, db[i][e] += dy;
                dw[i][e] = fmaf(dy, u, dw[i][e]);
            }
        }
        sum(v);
        const float along = mean_of(v[0], inv), level = LAYER ? mean_of(v[N - 1], inv) : 0.f;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int c = (i * lanes + lane) * V;
            if (c >= width) continue;
            forget(x[i]), forget(y[i]), forget(w[i]);
            float d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = (to_float(x[i].e[e]) - mean) * rstd, h = to_float(y[i].e[e]) * to_float(w[i].e[e]);
                d[e] = rstd * (h - level - u * along);
                if (dR) d[e] += to_float(r[i].e[e]);
            }
            store_cut<WHOLE, V>(dX + at, c, hidden, rounded<V>(d, T()));
        }
    }
    if (!want_w && !want_b) return;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (k == 0 ? !want_w : !want_b) continue;
        float* out = partial + ((int64_t)(k == 1 && want_w ? gridDim.x : 0) + blockIdx.x) * hidden;
        float(&d)[NA][V] = k == 0 ? dw : db;
        if constexpr (LANES) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) lds[row_of<LANES>() * (NA * V * LANES) + (i * LANES + lane) * V + e] = d[i][e];
            __syncthreads();
            for (int c = threadIdx.x; c < hidden; c += SMALL) {
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < ROWS; ++g) v += lds[g * (NA * V * LANES) + c];
                out[c] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = (i * lanes + lane) * V + e;
                    if (c < hidden) out[c] = d[i][e];
                }
        }
    }
}

// dw[c] += sum over the n rows of partial sums (db: the same, behind them), in 64 bits: rounded once, with what was there.  32 columns (a cache line)
// and 32 shares of the rows a workgroup.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float* partial, int n, int hidden, float* d0, float* d1)
{
    constexpr int COLS = 32, SHARES = 1024 / COLS, U = 8;
    __shared__ double part[SHARES][COLS];
    const int lane = threadIdx.x % COLS, w = threadIdx.x / COLS, c = blockIdx.x * COLS + lane;
    const float* p = partial + (int64_t)blockIdx.y * n * hidden + c;
    double v = 0;
    if (c < hidden) {
        int r = w;
        for (; r + (U - 1) * SHARES < n; r += U * SHARES) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = p[(int64_t)(r + u * SHARES) * hidden];
#pragma unroll
            for (int u = 0; u < U; ++u) v += x[u];
        }
        for (; r < n; r += SHARES) v += p[(int64_t)r * hidden];
    }
    part[w][lane] = v;
    __syncthreads();
    if (w || c >= hidden) return;
#pragma unroll
    for (int i = 1; i < SHARES; ++i) v += part[i][lane];
    float* d = blockIdx.y == 0 ? d0 : d1;
    d[c] = (float)(d[c] + v);
}

// f(Shape, threads) for a row of n accesses of elements of T.  Few accesses a lane keep registers free for rows under way; a wave's own row needs no
// barrier, but the backward's partial sums are then added up in LDS.  Measured with 2^27 elements in bf16, us: forward, 128 accesses, two waves 166, one
// with two 177; 1024 accesses, 8 waves with two 176, 16 with one 180.  Backward, 64 accesses, 64 lanes 180, 32 with two 192; 128 accesses,
// 64 lanes with two 193, two waves 201; 256 accesses, 4 waves 189, two with two 196; 640 accesses, 10 waves 201, 5 with two 302 (of 5 waves, fewer
// workgroups share a compute unit than registers would let).
template <int L, int N> struct Shape {
    static constexpr int lanes = L, accesses = N;
};
template <int N, class F> void wide(int n, F f) { f(Shape<0, N>(), 64 * ((n + 64 * N - 1) / (64 * N))); }
template <class T, class F> void fwd_shape(int n, F f)
{
    if (n <= 16) f(Shape<16, 1>(), SMALL);
    else if (n <= 32) f(Shape<32, 1>(), SMALL);
    else if (n <= 64) f(Shape<64, 1>(), SMALL);
    else if (n <= 512) wide<1>(n, f);
    else if (n <= 2048) wide<2>(n, f);
    else if constexpr (sizeof(T) == 4) wide<4>(n, f);
}
template <class T, class F> void bwd_shape(int n, F f)
{
    if (n <= 16) f(Shape<16, 1>(), SMALL);
    else if (n <= 32) f(Shape<32, 1>(), SMALL);
    else if (n <= 64) f(Shape<64, 1>(), SMALL);
    else if (n <= 128) f(Shape<64, 2>(), SMALL);
    else if (n <= 768) wide<1>(n, f);
    else if (n <= 2048) wide<2>(n, f);
    else if constexpr (sizeof(T) == 4) wide<4>(n, f);
}
// The backward's workgroups on rows of `hidden` elements of T, where there are rows enough.
template <class T> int bwd_most(int hidden)
{
    constexpr int V = 16 / sizeof(T);
    int most = 0;
    bwd_shape<T>((hidden + V - 1) / V, [&](auto shape, int threads) { most = bwd_groups(threads, decltype(shape)::accesses, hidden); });
    return most;
}
// f(std::true_type or false_type) for each of two rules
template <class F> void by_rule(bool a, bool b, F f)
{
    if (a && b) f(std::true_type(), std::true_type());
    else if (a) f(std::true_type(), std::false_type());
    else if (b) f(std::false_type(), std::true_type());
    else f(std::false_type(), std::false_type());
}

int check(int64_t rows, int hidden, int kind, int dtype)
{
    if (rows <= 0 || hidden <= 0) return fail(TW_INVALID, "rows and hidden must be positive");
    if (kind != FPDT_TW_RMSNORM && kind != FPDT_TW_LAYERNORM) return fail(TW_INVALID, "unknown kind %d", kind);
    if (dtype != FPDT_TW_F32 && dtype != FPDT_TW_BF16) return fail(TW_INVALID, "unknown dtype %d", dtype);
    if (hidden > MOST_HIDDEN || rows > INT32_MAX) return fail(TW_UNSUPPORTED, "hidden=%d beyond %d, or rows beyond the launch limits", hidden, MOST_HIDDEN);
    return TW_OK;
}

// An output may be an input's own memory (each element is read before it is written, by the same thread), not part of it.
int check_apart(const void* out, const char* name, const void* const* in, int n, size_t bytes)
{
    for (int i = 0; i < n; ++i)
        if (out && in[i] && out != in[i] && ranges_meet(out, bytes, in[i], bytes)) return fail(TW_INVALID, "%s overlaps another tensor without being it", name);
    return TW_OK;
}

unsigned groups_of(int64_t rows, int rows_at_once, int most)
{
    const int64_t n = (rows + rows_at_once - 1) / rows_at_once;
    return (unsigned)(n < most ? n : most);
}

template <class T>
void launch_fwd(const void* X, const void* R, const void* W, const void* B, void* S, void* Y, float* stats, int64_t rows, int hidden, int kind, float eps,
                hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    auto t = [](const void* p) { return static_cast<const T*>(p); };
    fwd_shape<T>((hidden + V - 1) / V, [&](auto shape, int threads) {
        constexpr int L = decltype(shape)::lanes, N = decltype(shape)::accesses;
        const unsigned grid = groups_of(rows, L ? SMALL / (L ? L : 1) : 1, 1 << 21);
        by_rule(kind == FPDT_TW_LAYERNORM, hidden % V == 0, [&](auto layer, auto whole) {
            norm_fwd_kernel<T, L, N, decltype(layer)::value, decltype(whole)::value>
                <<<grid, threads, 0, st>>>(t(X), t(R), t(W), t(B), static_cast<T*>(S), static_cast<T*>(Y), stats, rows, hidden, 1. / hidden, eps);
        });
    });
}

template <class T>
void launch_bwd(const void* S, const void* W, const float* stats, const void* dY, const void* dR, void* dX, float* dW, float* dB, int64_t rows, int hidden,
                int kind, float* partial, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    auto t = [](const void* p) { return static_cast<const T*>(p); };
    bwd_shape<T>((hidden + V - 1) / V, [&](auto shape, int threads) {
        constexpr int L = decltype(shape)::lanes, N = decltype(shape)::accesses;
        const unsigned grid = groups_of(rows, L ? SMALL / (L ? L : 1) : 1, bwd_most<T>(hidden));
        by_rule(kind == FPDT_TW_LAYERNORM, hidden % V == 0, [&](auto layer, auto whole) {
            norm_bwd_kernel<T, L, N, decltype(layer)::value, decltype(whole)::value>
                <<<grid, threads, 0, st>>>(t(S), t(W), stats, t(dY), t(dR), static_cast<T*>(dX), partial, rows, hidden, 1. / hidden, dW, dB);
        });
        if (dW || dB)
            norm_sums_kernel<<<dim3((hidden + 31) / 32, dW && dB ? 2 : 1), 1024, 0, st>>>(partial, (int)grid, hidden, dW ? dW : dB, dB);
    });
}

}  // namespace

extern "C" {

int fpdt_tw_norm_fwd(const void* X, const void* R, const void* W, const void* B, void* S, void* Y, float* stats, int64_t rows, int hidden, int kind,
                     float eps, int dtype, void* stream)
{
    clear_error();
    if (!X || !W || !Y) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check(rows, hidden, kind, dtype);
    if (rc != TW_OK) return rc;
    if (S && !R) return fail(TW_INVALID, "S is the sum of X and R: R is NULL");
    if (B && kind == FPDT_TW_RMSNORM) return fail(TW_INVALID, "RMSNORM has no bias");
    if (!std::isfinite(eps) || eps < 0) return fail(TW_INVALID, "eps must be finite and not negative");
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, bytes = (size_t)rows * hidden * size;
    const void* every[6] = {X, R, W, B, S, Y};
    for (const void* p : every)
        if (misaligned(p, size)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    if (misaligned(stats, 4)) return fail(TW_INVALID, "stats is not aligned to its elements");
    const void* in[2] = {X, R};
    if ((rc = check_apart(S, "S", in, 2, bytes)) != TW_OK || (rc = check_apart(Y, "Y", in, 2, bytes)) != TW_OK) return rc;
    if (S && ranges_meet(S, bytes, Y, bytes)) return fail(TW_INVALID, "S and Y overlap");
    const void* row[2] = {W, B};
    const size_t nstats = (size_t)rows * 4 * (kind == FPDT_TW_LAYERNORM ? 2 : 1);
    for (const void* p : row)
        if (p && (ranges_meet(S, S ? bytes : 0, p, hidden * size) || ranges_meet(Y, bytes, p, hidden * size))) return fail(TW_INVALID, "an output overlaps W or B");
    for (const void* p : every)
        if (stats && p && ranges_meet(stats, nstats, p, p == W || p == B ? hidden * size : bytes)) return fail(TW_INVALID, "stats overlaps a tensor");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (size == 4) launch_fwd<float>(X, R, W, B, S, Y, stats, rows, hidden, kind, eps, st);
    else launch_fwd<uint16_t>(X, R, W, B, S, Y, stats, rows, hidden, kind, eps, st);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

size_t fpdt_tw_norm_bwd_workspace_bytes(int64_t rows, int hidden, int kind)
{
    if (rows <= 0 || hidden <= 0 || hidden > MOST_HIDDEN || rows > INT32_MAX || (kind != FPDT_TW_RMSNORM && kind != FPDT_TW_LAYERNORM)) return 0;
    // one row of partial sums per workgroup, of the type that has more of them, and never more workgroups than rows
    const int f = bwd_most<float>(hidden), b = bwd_most<uint16_t>(hidden);
    return (size_t)groups_of(rows, 1, f > b ? f : b) * hidden * 4 * (kind == FPDT_TW_LAYERNORM ? 2 : 1);
}

int fpdt_tw_norm_bwd(const void* S, const void* W, const float* stats, const void* dY, const void* dR, void* dX, float* dW, float* dB, int64_t rows,
                     int hidden, int kind, int dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    if (!S || !W || !stats || !dY || !dX) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check(rows, hidden, kind, dtype);
    if (rc != TW_OK) return rc;
    if (dB && kind == FPDT_TW_RMSNORM) return fail(TW_INVALID, "RMSNORM has no bias");
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, bytes = (size_t)rows * hidden * size;
    const void* every[5] = {S, W, dY, dR, dX};
    for (const void* p : every)
        if (misaligned(p, size)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    if (misaligned(stats, 4) || misaligned(dW, 4) || misaligned(dB, 4)) return fail(TW_INVALID, "stats, dW or dB is not aligned to its elements");
    const size_t need = dW || dB ? fpdt_tw_norm_bwd_workspace_bytes(rows, hidden, kind) : 0;
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 256)))
        return fail(TW_WORKSPACE, "workspace NULL, misaligned or too small (%zu < %zu bytes)", workspace_bytes, need);
    const void* in[3] = {S, dY, dR};
    if ((rc = check_apart(dX, "dX", in, 3, bytes)) != TW_OK) return rc;
    const size_t nstats = (size_t)rows * 4 * (kind == FPDT_TW_LAYERNORM ? 2 : 1), ncol = (size_t)hidden * 4;
    if (ranges_meet(dX, bytes, W, hidden * size) || ranges_meet(dX, bytes, stats, nstats)) return fail(TW_INVALID, "dX overlaps W or stats");
    if (dW && dB && ranges_meet(dW, ncol, dB, ncol)) return fail(TW_INVALID, "dW and dB overlap");
    // what is written besides dX meets nothing that is read, or dX
    struct Out {
        const void* p;
        size_t n;
    } outs[3] = {{dW, dW ? ncol : 0}, {dB, dB ? ncol : 0}, {workspace, need}};
    for (const Out& o : outs) {
        for (const void* p : every)
            if (p && ranges_meet(o.p, o.n, p, p == W ? hidden * size : bytes)) return fail(TW_INVALID, "dW, dB or the workspace overlaps a tensor");
        if (ranges_meet(o.p, o.n, stats, nstats)) return fail(TW_INVALID, "dW, dB or the workspace overlaps stats");
    }
    if (ranges_meet(workspace, need, dW, dW ? ncol : 0) || ranges_meet(workspace, need, dB, dB ? ncol : 0)) return fail(TW_INVALID, "the workspace overlaps dW or dB");
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* partial = static_cast<float*>(workspace);
    if (size == 4) launch_bwd<float>(S, W, stats, dY, dR, dX, dW, dB, rows, hidden, kind, partial, st);
    else launch_bwd<uint16_t>(S, W, stats, dY, dR, dX, dW, dB, rows, hidden, kind, partial, st);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // extern "C"
