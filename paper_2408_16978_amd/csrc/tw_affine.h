// What the products with something behind them (tw_affine.hip) and those of the experts (tw_experts_gemm.hip) share.
#pragma once
#include <initializer_list>

#include "../../include/fpdt_tokenwise.h"
#include "tw_act.h"
#include "tw_common.h"
#include "tw_gemm_tile.h"

namespace fpdt_tw {
namespace {

constexpr int MOST_EXPERTS = 1024;
constexpr int MOST_WIDTH = 1 << 22;              // a lane's offset within a tile is kept in 32 bits

// What is done behind a product, in fp32.  Pointers are to the first of the product's rows (B: columns).
template <int ACT> struct Epilogue {
    static constexpr bool any = true;
    const uint16_t *B, *R;
    uint16_t *Z, *Y;
    bool times;  // R multiplies the activation, otherwise it is added to it
    bool wide;   // rows come in aligned pieces of 16 bytes in all of them
    __device__ __forceinline__ float act(float z) const { return act_of<ACT>(z); }
    __device__ __forceinline__ void one(float z, int64_t at) const
    {
        if (Z) Z[at] = from_float<uint16_t>(z);
        float y = act(z);
        if (R) y = times ? y * to_float(R[at]) : y + to_float(R[at]);
        Y[at] = from_float<uint16_t>(y);
    }
    // Four columns of row m from n on (fewer at the end of a row of N), without their bias yet.
    __device__ __forceinline__ void four(floatx4 v, int m, int n, int N) const
    {
        const int64_t c = (int64_t)m * N + n;
        if (wide) {  // (N is a multiple of 8)
            if (B) {
                const auto b = load<4>(B + n);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] += to_float(b.e[r]);
            }
            float y[4];
            if (Z) {
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = v[r];
                store(Z + c, rounded<4>(y, uint16_t()));
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = act(v[r]);
            if (R) {
                const auto j = load<4>(R + c);
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = times ? y[r] * to_float(j.e[r]) : y[r] + to_float(j.e[r]);
            }
            store(Y + c, rounded<4>(y, uint16_t()));
        } else {
            for (int r = 0; r < 4 && n + r < N; ++r) one(v[r] + (B ? to_float(B[n + r]) : 0.f), c + r);
        }
    }
};

// ---- few rows -------------------------------------------------------------------------------
// The product of M <= 16 MT rows with 16 columns (rows of W) from n0 on, and what is behind it, by one workgroup of FEW_WAVES waves: a wave takes a
// range of k, fragments straight from memory (no other workgroup reads these rows of W; those of X come from L2), and the
// waves' sums are added in LDS.  Bound by the memory, that is by the bytes under way: the fragments of the next U units are requested before
// the MFMAs of these, and there is no barrier but the last.  16 rows (n_in x n_out), 1 GB of weights in turn, so that they come from HBM, us: 4096 x 4096 10.8-11.4
// (tiles of 64 x 256 in 16 splits and their sums 19.7; 3.1 TB/s of weights), 1024 x 1024 4.6 (10.5), 2560 x 10240 20.7 (22.1), but 4096 x 14336 35.6 (34.2).  Over three
// sets in turn, which the caches hold in part, 32 columns a workgroup, which read X half as often, took 15.5 for 11.4, 5.1 for 4.3, 21.7 for 20.4 and 30.9 for 35.3; loads
// of W past the caches, which fetch a line for each half of it, 11.6, 4.5, 22.7 and 36.9.
constexpr int FEW_WAVES = 8, FEW_ROWS = 64, FEW_COLS = 16;
template <int ACT, int MT> __device__ __forceinline__ void few_rows(float* sums, const uint16_t* X, const uint16_t* W, int K, int M, int N, int n0, const Epilogue<ACT>& behind)
{
    constexpr int U = 2;  // units of 64 k
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fk = 8 * (lane >> 4);
    // this wave's part of k, in units of 64
    const int units = (K + 63) / 64, each = (units + FEW_WAVES - 1) / FEW_WAVES, first = wave * each, last = first + each < units ? first + each : units;
    // rows behind the operands are read as the last one: their products are not stored
    const uint16_t *w = W + (int64_t)(n0 + fr < N ? n0 + fr : N - 1) * K + fk + 64 * first, *x[MT];
    floatx4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        x[i] = X + (int64_t)(16 * i + fr < M ? 16 * i + fr : M - 1) * K + fk + 64 * first;
        acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    struct Some {
        bf16x8 a[U][2], b[U][2][MT];
    };
    auto fetch = [&](Some& s, int k0, auto whole_tag) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole_tag)::value;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 64 * u + 32 * h;
                const bool in = WHOLE || (64 * first + k < 64 * last && 64 * first + k + fk < K);  // (K is a multiple of 8)
                s.a[u][h] = in ? *reinterpret_cast<const bf16x8*>(w + k) : bf16x8{};
#pragma unroll
                for (int i = 0; i < MT; ++i) s.b[u][h][i] = in ? *reinterpret_cast<const bf16x8*>(x[i] + k) : bf16x8{};
            }
    };
    auto add = [&](const Some& s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s.a[u][h], s.b[u][h][i], acc[i], 0, 0, 0);
    };
    const int mine = (last < K / 64 ? last : K / 64) - first, whole = mine > 0 ? mine / U : 0;  // this wave's whole units, and U at a time
    Some s0, s1;
    if (whole > 0) {
        fetch(s0, 0, std::true_type{});
        int i = 0;
        for (; i + 2 < whole; i += 2) {  // (nothing is conditional in here: a wait counts what is under way)
            fetch(s1, 64 * U * (i + 1), std::true_type{});
            __builtin_amdgcn_sched_barrier(0);
            add(s0);
            fetch(s0, 64 * U * (i + 2), std::true_type{});
            __builtin_amdgcn_sched_barrier(0);
            add(s1);
        }
        if (i + 1 < whole) {
            fetch(s1, 64 * U * (i + 1), std::true_type{});
            add(s0);
            add(s1);
        } else {
            add(s0);
        }
    }
    if (first + U * whole < last) {
        fetch(s0, 64 * U * whole, std::false_type{});
        add(s0);
    }
    // a lane has columns 4 (lane / 16) .. + 3 of row lane % 16
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<floatx4*>(sums + ((wave * MT + i) * 64 + lane) * 4) = acc[i];
    __syncthreads();
    for (int t = threadIdx.x; t < MT * 64; t += FEW_WAVES * 64) {
        floatx4 v = *reinterpret_cast<const floatx4*>(sums + t * 4);
#pragma unroll
        for (int s = 1; s < FEW_WAVES; ++s) v += *reinterpret_cast<const floatx4*>(sums + (s * MT * 64 + t) * 4);
        const int m = 16 * (t / 64) + t % 16, n = n0 + 4 * (t % 64 / 16);
        if (m < M && n < N) behind.four(v, m, n, N);
    }
}
// Every 16 columns read X anew: it pays while that is not much.  Measured with weights from HBM, us, few_rows and tiles: 1 row, 4096 x 14336 25.7 and 31.6; 32 rows, 4096 x
// 4096 14.3 and 19.4, 14336 x 4096 44.9 and 36.3; 64 rows, 1024 x 1024 7.4 and 11.0, 4096 x 4096 22.4 and 19.8; 16 rows, 14336 x 4096 34.9 and 36.2, 4096 x 14336 35.6 and
// 34.2.
inline bool few_pays(int64_t rows, int64_t weights) { return rows * weights <= (int64_t)16 * 34 << 20; }
template <int MT> constexpr int few_lds = FEW_WAVES * MT * 64 * 4;  // floats

// Where expert e's rows begin and end, whatever the offsets say within the rows that there are.
__device__ __forceinline__ int offset_of(const int32_t* offsets, int e, int rows)
{
    const int o = offsets[e];
    return o < 0 ? 0 : o < rows ? o : rows;
}

// ---- host side ----------------------------------------------------------------------------
// f(Int<act>) for an activation that was checked
template <class F> void by_act(int act, F f)
{
    if (act == FPDT_TW_ACT_GELU) f(Int<FPDT_TW_ACT_GELU>());
    else if (act == FPDT_TW_ACT_SILU) f(Int<FPDT_TW_ACT_SILU>());
    else f(Int<FPDT_TW_ACT_NONE>());
}
// f(Int<WMT>, Int<WNT>) for the tiles that plans have
template <class F> void by_tile(int wmt, int wnt, F f)
{
    if (wnt == 2) f(Int<2>(), Int<2>());
    else if (wmt == 4) f(Int<4>(), Int<4>());
    else if (wmt == 3) f(Int<3>(), Int<4>());
    else if (wmt == 2) f(Int<2>(), Int<4>());
    else f(Int<1>(), Int<4>());
}

int check_sizes(int64_t rows, int n_in, int n_out)
{
    if (rows <= 0 || n_in <= 0 || n_out <= 0) return fail(TW_INVALID, "rows, n_in and n_out must be positive");
    if (n_in > MOST_WIDTH || n_out > MOST_WIDTH || rows > INT32_MAX) return fail(TW_UNSUPPORTED, "sizes beyond the launch limits");
    return TW_OK;
}
int check_kind(int act, int join)
{
    if (act < FPDT_TW_ACT_NONE || act > FPDT_TW_ACT_SILU) return fail(TW_INVALID, "unknown activation %d", act);
    if (join != FPDT_TW_JOIN_ADD && join != FPDT_TW_JOIN_TIMES) return fail(TW_INVALID, "unknown join %d", join);
    return TW_OK;
}

// A tensor of a call: what it is called, its bytes, whether it is written.
struct Arg {
    const char* name;
    const void* p;
    size_t bytes;
    bool written;
};
// Two of them that overlap, one at least written, are refused, but for `same`: pairs that may be one tensor (not a part of it).
int check_apart(const Arg* a, int n, const int (*same)[2], int nsame)
{
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j) {
            if (!a[i].p || !a[j].p || !(a[i].written || a[j].written) || !ranges_meet(a[i].p, a[i].bytes, a[j].p, a[j].bytes)) continue;
            bool may = false;
            for (int k = 0; k < nsame; ++k) may = may || (a[i].p == a[j].p && same[k][0] == i && same[k][1] == j);
            if (!may) return fail(TW_INVALID, "%s and %s overlap", a[i].name, a[j].name);
        }
    return TW_OK;
}

// Do rows of n elements come in aligned pieces of 16 bytes in all of these tensors?
bool all_wide(int n, std::initializer_list<const void*> every)
{
    for (const void* p : every)
        if (misaligned(p, 16)) return false;
    return n % 8 == 0;
}

}  // namespace
}  // namespace fpdt_tw
