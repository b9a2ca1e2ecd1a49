// The products of the experts' backward (include/fpdt_tokenwise.h: fpdt_tw_experts_linear_bwd).
//
//     dx = dy W,   dW += dy^T x                              (for each expert's rows)
//
// 64 experts, 30000 rows, 2048 x 1536: dx 200 us, 0.94 PFLOP/s (24 stages of k a tile, and an epilogue each); dW 372 us, bound by its sums in fp32, 1.6 GB read and written,
// which several workgroups a compute unit (tiles of 64 x 256 and 128 x 128) did not hide better (447 and 414).
#include "tw_experts_gemm.h"

namespace fpdt_tw {
namespace {

// dX of an expert's rows = dY W
template <int WMT, int WNT>
__global__ __launch_bounds__(NTHREAD, 1) void experts_dx_kernel(const uint16_t* dY, const uint16_t* W, uint16_t* dX, int n_in, int n_out, Groups g)
{
    __shared__ __attribute__((aligned(256))) u32x4 ring[ring_bytes(WMT, WNT) / 16];
    GroupTile t;
    if (!find_group(g, 64 * WMT, ((unsigned)n_in + 64 * WNT - 1) / (64 * WNT), t)) return;
    const int skip = (int)fpdt::uniform((unsigned)t.tile_m) * (64 * WMT), left = t.rows - skip, tile_n = (int)fpdt::uniform((unsigned)t.tile_n);
    const int64_t first = (int64_t)t.first + skip;
    const Operand a = {dY + first * n_out, n_out, left}, b = {W + (int64_t)t.expert * n_out * n_in, n_in, n_in};
    by_rows<WMT>(left, [&](auto w) __attribute__((always_inline)) {
        product_tile<false, true, false, false, decltype(w)::value, WNT>(ring, a, b, n_out, dX + first * n_in, n_in, left, n_in, 0, tile_n, 0, n_out / STAGE_K, false, Whole(),
                                                                        Nothing());
    });
}

// dW of an expert += dY^T X over its rows
template <int WMT, int WNT>
__global__ __launch_bounds__(NTHREAD, 1) void experts_dw_kernel(const uint16_t* X, const uint16_t* dY, float* dW, int n_in, int n_out, Groups g)
{
    __shared__ __attribute__((aligned(256))) u32x4 ring[ring_bytes(WMT, WNT) / 16];
    const unsigned tiles_n = ((unsigned)n_in + 64 * WNT - 1) / (64 * WNT), tiles_m = ((unsigned)n_out + 64 * WMT - 1) / (64 * WMT);
    const unsigned total = tiles_m * tiles_n * (unsigned)g.experts, run = (total + 7) / 8, xcd = blockIdx.x % 8, turn = blockIdx.x / 8, id = xcd * run + turn;
    if (turn >= run || id >= total) return;
    const unsigned e = id / (tiles_m * tiles_n);
    const int first = (int)fpdt::uniform((unsigned)offset_of(g.offsets, (int)e, g.rows)), last = (int)fpdt::uniform((unsigned)offset_of(g.offsets, (int)e + 1, g.rows));
    if (last <= first) return;
    int tile_m, tile_n;
    tile_of(id - e * (tiles_m * tiles_n), tiles_m, tiles_n, tile_m, tile_n);
    const Operand a = {dY + (int64_t)first * n_out, n_out, n_out}, b = {X + (int64_t)first * n_in, n_in, n_in};
    product_tile<true, true, true, true, WMT, WNT>(ring, a, b, last - first, dW + (int64_t)e * n_out * n_in, n_in, n_out, n_in, tile_m, tile_n, 0, (last - first) / STAGE_K, false,
                                                   Whole(), Nothing());
}

// The weights' gradient: as many tiles whatever the offsets, over the rows of an expert.
GroupPlan plan_weights(int64_t rows, int experts, int n_in, int n_out)
{
    static const int shapes[][2] = {{4, 4}, {3, 4}, {1, 4}, {2, 2}};
    GroupPlan best = {4, 4, 0};
    double best_cost = 0;
    const int64_t busy = rows < experts ? rows : experts, K = (rows + busy - 1) / busy;
    for (const auto& sh : shapes) {
        const int64_t each = (int64_t)((n_in + 64 * sh[1] - 1) / (64 * sh[1])) * ((n_out + 64 * sh[0] - 1) / (64 * sh[0])), tiles = each * busy;
        if (each * experts > MOST_TILES) continue;
        const int slots = sh[0] * sh[1] <= 4 ? 512 : 256;
        const double c = launch_cost(sh[0], sh[1], (double)(tiles / slots * slots), (double)(tiles % slots), 1, (int)((K < SK ? SK : K) / SK));
        if (best_cost == 0 || c < best_cost) best = {sh[0], sh[1], each * experts}, best_cost = c;
    }
    return best;
}

}  // namespace
}  // namespace fpdt_tw

using namespace fpdt_tw;

extern "C" {

int fpdt_tw_experts_linear_bwd(const void* X, const void* W, const void* dY, void* dX, float* dW, const int32_t* offsets, int64_t rows, int experts, int n_in,
                               int n_out, void* stream)
{
    clear_error();
    if (!X || !W || !dY || !offsets) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_experts(rows, experts, n_in, n_out);
    if (rc != TW_OK) return rc;
    if (misaligned(X, 16) || misaligned(W, 16) || misaligned(dY, 16)) return fail(TW_INVALID, "X, W and dY must be 16-byte aligned");
    if (misaligned(dX, 2) || misaligned(dW, 4) || misaligned(offsets, 4)) return fail(TW_INVALID, "dX, dW or offsets is not aligned to its elements");
    const size_t weights = (size_t)experts * n_in * n_out;
    const Arg args[] = {{"X", X, (size_t)rows * n_in * 2, false}, {"W", W, weights * 2, false}, {"dY", dY, (size_t)rows * n_out * 2, false},
                        {"dX", dX, (size_t)rows * n_in * 2, true}, {"dW", dW, weights * 4, true}, {"offsets", offsets, (size_t)(experts + 1) * 4, false}};
    if ((rc = check_apart(args, 6, nullptr, 0)) != TW_OK) return rc;
    const GroupPlan px = plan_groups(rows, experts, n_in, n_out), pw = plan_weights(rows, experts, n_in, n_out);
    if ((dX && px.tiles == 0) || (dW && pw.tiles == 0)) return fail(TW_UNSUPPORTED, "product beyond the launch limits");
    const Groups g = {offsets, experts, (int)rows};
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto t = [](const void* p) { return static_cast<const uint16_t*>(p); };
    if (dX)
        by_group_tile(px, [&](auto wm, auto wn) {
            experts_dx_kernel<decltype(wm)::value, decltype(wn)::value><<<grid_of(px.tiles), NTHREAD, 0, st>>>(t(dY), t(W), static_cast<uint16_t*>(dX), n_in, n_out, g);
        });
    if (dW)
        by_group_tile(pw, [&](auto wm, auto wn) {
            experts_dw_kernel<decltype(wm)::value, decltype(wn)::value><<<grid_of(pw.tiles), NTHREAD, 0, st>>>(t(X), t(dY), dW, n_in, n_out, g);
        });
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // extern "C"
