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
};

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
