// What the experts' products (tw_experts_gemm.hip) and those of their backward (tw_experts_gemm_bwd.hip) share: where a workgroup's tile is, and plans.
//
// An expert's rows are neighbours, from offsets[e] on; offsets are known to the device alone, so a launch has as many workgroups as the
// rows could need, and each finds its expert and tile from them.
#pragma once
#include <cmath>

#include "tw_affine.h"

namespace fpdt_tw {
namespace {

struct Groups {
    const int32_t* offsets;
    int experts, rows;
};

// Tile number `turn` of this XCD's share, of all experts' tiles of tm rows in their order: the expert, its rows, and the tile among its own.
struct GroupTile {
    int expert, first, rows, tile_m, tile_n;
};
__device__ __forceinline__ unsigned tiles_of(int rows, int tm) { return ((unsigned)rows + (unsigned)tm - 1) / (unsigned)tm; }
__device__ __forceinline__ bool find_group(const Groups& g, int tm, unsigned tiles_n, GroupTile& at)
{
    // a lane counts the tile rows of `per` neighbouring experts, of which it keeps the first one's rows
    const int lane = threadIdx.x & 63, per = (g.experts + 63) / 64, e0 = lane * per;
    auto begin_of = [&](int e) { return offset_of(g.offsets, e < g.experts ? e : g.experts, g.rows); };
    const int own = begin_of(e0), next = begin_of(e0 + 1), own_rows = next > own ? next - own : 0;
    unsigned mine = tiles_of(own_rows, tm);
    for (int i = 1, from = next; i < per; ++i) {
        const int to = begin_of(e0 + i + 1);
        mine += to > from ? tiles_of(to - from, tm) : 0u;
        from = to;
    }
    unsigned upto = mine;  // those of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned v = __shfl_up(upto, d, 64);
        if (lane >= d) upto += v;
    }
    const unsigned total = (unsigned)__builtin_amdgcn_readlane((int)upto, 63) * tiles_n;
    const unsigned xcd = blockIdx.x % 8, turn = blockIdx.x / 8, run = (total + 7) / 8, id = xcd * run + turn;
    if (turn >= run || id >= total) return false;  // whole workgroup, before any barrier
    const int owner = __builtin_ctzll(__ballot(upto * tiles_n > id));
    unsigned base = (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), owner);
    int e = owner * per, first = __builtin_amdgcn_readlane(own, owner), rows = __builtin_amdgcn_readlane(own_rows, owner);
    unsigned tiles = tiles_of(rows, tm);
    while ((base + tiles) * tiles_n <= id && e + 1 < g.experts) {  // (not with 64 experts and fewer)
        base += tiles;
        first = begin_of(++e);
        const int end = begin_of(e + 1);
        rows = end > first ? end - first : 0;
        tiles = tiles_of(rows, tm);
    }
    if (id - base * tiles_n >= tiles * tiles_n) return false;  // (offsets that do not ascend)
    at.expert = (int)fpdt::uniform((unsigned)e);
    at.first = (int)fpdt::uniform((unsigned)first);
    at.rows = (int)fpdt::uniform((unsigned)rows);
    tile_of_few(fpdt::uniform(id - base * tiles_n), fpdt::uniform(tiles), tiles_n, at.tile_m, at.tile_n);
    return true;
}

// No tile is divided.
struct Whole {
    __device__ __forceinline__ float* operator()(size_t) const { return nullptr; }
};

// f(Int<WMT'>, tile): the tile of WMT' x 64 rows that a workgroup of `left` rows needs, so that an expert's last rows do not cost a whole tile.
template <int WMT, class F> __device__ __forceinline__ void by_rows(int left, F f)
{
    if constexpr (WMT > 1) {
        if (left <= 64 * (WMT - 1)) return by_rows<WMT - 1>(left, f);
    }
    f(Int<WMT>());
}

// Tiles for experts' products of about rows / experts rows each (a spread of them: 0.6 to 1.4 times that): the cheapest by launch_cost's terms, clocks of a
// tile, counting an expert's last tile as what by_rows makes of it.  Few rounds are counted whole, of many half a round is lost at the end.
// Measured, us: 64 experts of 64 rows, 2048 x 1536, tiles of 256 x 256 (and what they become) 108, of 64 x 256, two workgroups a compute unit, 119; 8 of 37
// rows, 4096 x 14336, 191 and 161; 8 of 250 rows, 1024 x 1024, 25 and 14, of 128 x 128 11.
struct GroupPlan {
    int wmt, wnt;
    int64_t tiles;  // at most, whatever the offsets; 0: more in every tile than a launch has
};
// Of a launch of 2^32 threads and more, those beyond do not run, without an error.  (A grid is rounded up to a multiple of 8.)
constexpr int64_t MOST_TILES = ((int64_t)1 << 32) / NTHREAD - 8;
double tile_clocks(int wm, int wn, bool two, int steps)
{
    const double mfma = two ? 161. * wm * wn + 158. : 64. * wm * wn + 116., copies = (two ? 175. : 85.) * (wm + wn);
    return steps * (mfma > copies ? mfma : copies) + (two ? 8100. + 1385. * wm * wn : 6900. + 1630. * wm * wn);
}
GroupPlan plan_groups(int64_t rows, int experts, int N, int K)
{
    static const int shapes[][2] = {{4, 4}, {3, 4}, {1, 4}, {2, 2}};
    GroupPlan best = {4, 4, 0};
    double best_cost = 0;
    const int64_t busy = rows < experts ? rows : experts;
    const int steps = (K < SK ? SK : K) / SK;
    for (const auto& sh : shapes) {
        const bool two = sh[0] * sh[1] <= 4;
        const int64_t tiles_n = (N + 64 * sh[1] - 1) / (64 * sh[1]), tm = 64 * sh[0], tiles = (rows / tm + busy) * tiles_n;
        if (tiles > MOST_TILES) continue;
        double n = 0, work = 0;
        for (int k = 0; k < 5; ++k) {
            const double some = (0.6 + 0.2 * k) * (double)rows / (double)busy;
            const int64_t r = some < 1 ? 1 : (int64_t)some, last = r % tm;
            const double share = (double)(busy * tiles_n) / 5;
            n += share * (double)(r / tm + (last > 0));
            work += share * ((double)(r / tm) * tile_clocks(sh[0], sh[1], two, steps) + (last > 0 ? tile_clocks((int)((last + 63) / 64), sh[1], two, steps) : 0));
        }
        const double rounds = n / (two ? 512 : 256), c = work / n * (rounds < 3 ? std::ceil(rounds) : rounds + 0.5) * (two && n <= 256 ? 0.56 : 1.);
        if (best_cost == 0 || c < best_cost) best = {sh[0], sh[1], tiles}, best_cost = c;
    }
    return best;
}
// f(Int<WMT>, Int<WNT>) for the tiles that these plans have
template <class F> void by_group_tile(const GroupPlan& p, F f)
{
    if (p.wnt == 2) f(Int<2>(), Int<2>());
    else if (p.wmt == 4) f(Int<4>(), Int<4>());
    else if (p.wmt == 3) f(Int<3>(), Int<4>());
    else f(Int<1>(), Int<4>());
}
unsigned grid_of(int64_t tiles) { return 8u * (unsigned)((tiles + 7) / 8); }

int check_experts(int64_t rows, int experts, int n_in, int n_out)
{
    int rc = check_sizes(rows, n_in, n_out);
    if (rc != TW_OK) return rc;
    if (experts <= 0) return fail(TW_INVALID, "experts must be positive");
    if (experts > MOST_EXPERTS) return fail(TW_UNSUPPORTED, "experts=%d beyond %d", experts, MOST_EXPERTS);
    if (n_in % 8 || n_out % 8) return fail(TW_UNSUPPORTED, "n_in=%d and n_out=%d of experts must be multiples of 8", n_in, n_out);
    return TW_OK;
}

}  // namespace
}  // namespace fpdt_tw
