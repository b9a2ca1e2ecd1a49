// The experts' products (include/fpdt_tokenwise.h: fpdt_tw_experts_affine_fwd).
//
//     z = x W^T + b,   y = act(z) + r  or  act(z) r          (W, b: of the row's expert)
//
// Bound by the matrix cores as the dense product is (61% of the cycles; 16384 rows of 8 experts, 4096 x 14336, bare 1540 us, the dense product 1282), and with few rows
// by the weights' bytes.  What the experts cost: rounds of tiles that are partly empty, and weights that no other rows share.
#include "tw_experts_gemm.h"

namespace fpdt_tw {
namespace {

// Rows of X and of what is behind the product begin at the tile's own.
template <int ACT, int WMT, int WNT>
__global__ __launch_bounds__(NTHREAD, 1) void experts_affine_kernel(const uint16_t* X, const uint16_t* W, int n_in, int n_out, Groups g, Epilogue<ACT> behind)
{
    __shared__ __attribute__((aligned(256))) u32x4 ring[ring_bytes(WMT, WNT) / 16];
    GroupTile t;
    if (!find_group(g, 64 * WMT, ((unsigned)n_out + 64 * WNT - 1) / (64 * WNT), t)) return;
    const int skip = (int)fpdt::uniform((unsigned)t.tile_m) * (64 * WMT), left = t.rows - skip, tile_n = (int)fpdt::uniform((unsigned)t.tile_n);
    const int64_t first = (int64_t)t.first + skip, out = first * n_out;
    const Operand a = {X + first * n_in, n_in, left}, b = {W + (int64_t)t.expert * n_out * n_in, n_in, n_out};
    if (behind.B) behind.B += (int64_t)t.expert * n_out;
    if (behind.R) behind.R += out;
    if (behind.Z) behind.Z += out;
    behind.Y += out;
    by_rows<WMT>(left, [&](auto w) __attribute__((always_inline)) {
        product_tile<false, false, false, false, decltype(w)::value, WNT>(ring, a, b, n_in, nullptr, n_out, left, n_out, 0, tile_n, 0, n_in / STAGE_K, false, Whole(), behind);
    });
}

// Few rows in all, and so of each expert (blockIdx.y): 16 at a time.
template <int ACT> __global__ __launch_bounds__(FEW_WAVES * 64) void experts_few_kernel(const uint16_t* X, const uint16_t* W, int n_in, int n_out, Groups g, Epilogue<ACT> behind)
{
    __shared__ __attribute__((aligned(16))) float sums[few_lds<1>];
    const int e = blockIdx.y, first = offset_of(g.offsets, e, g.rows), rows = offset_of(g.offsets, e + 1, g.rows) - first;
    if (rows <= 0) return;
    if (behind.B) behind.B += (int64_t)e * n_out;
    for (int m = 0; m < rows; m += 16) {
        const int64_t out = (int64_t)(first + m) * n_out;
        Epilogue<ACT> here = behind;
        if (here.R) here.R += out;
        if (here.Z) here.Z += out;
        here.Y += out;
        if (m) __syncthreads();  // the sums of the rows before have been read
        few_rows<ACT, 1>(sums, X + (int64_t)(first + m) * n_in, W + (int64_t)e * n_out * n_in, n_in, rows - m < 16 ? rows - m : 16, n_out, blockIdx.x * FEW_COLS, here);
    }
}

}  // namespace
}  // namespace fpdt_tw

using namespace fpdt_tw;

extern "C" {

int fpdt_tw_experts_affine_fwd(const void* X, const void* W, const void* B, const void* R, void* Z, void* Y, const int32_t* offsets, int64_t rows, int experts,
                               int n_in, int n_out, int act, int join, void* stream)
{
    clear_error();
    if (!X || !W || !Y || !offsets) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_experts(rows, experts, n_in, n_out);
    if (rc != TW_OK || (rc = check_kind(act, join)) != TW_OK) return rc;
    if (join == FPDT_TW_JOIN_TIMES && !R) return fail(TW_INVALID, "JOIN_TIMES needs R");
    for (const void* p : {B, R, (const void*)Z, (const void*)Y})
        if (misaligned(p, 2)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    if (misaligned(X, 16) || misaligned(W, 16)) return fail(TW_INVALID, "X and W must be 16-byte aligned");
    if (misaligned(offsets, 4)) return fail(TW_INVALID, "offsets is not aligned to its elements");
    const size_t out = (size_t)rows * n_out * 2;
    const Arg args[] = {{"X", X, (size_t)rows * n_in * 2, false}, {"W", W, (size_t)experts * n_in * n_out * 2, false}, {"B", B, (size_t)experts * n_out * 2, false},
                        {"R", R, out, false}, {"Z", Z, out, true}, {"Y", Y, out, true}, {"offsets", offsets, (size_t)(experts + 1) * 4, false}};
    const int same[][2] = {{3, 5}};
    if ((rc = check_apart(args, 7, same, 1)) != TW_OK) return rc;
    const GroupPlan plan = plan_groups(rows, experts, n_out, n_in);
    if (plan.tiles == 0) return fail(TW_UNSUPPORTED, "product beyond the launch limits");
    const Groups g = {offsets, experts, (int)rows};
    hipStream_t st = static_cast<hipStream_t>(stream);
    by_act(act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        const Epilogue<ACT> behind = {static_cast<const uint16_t*>(B), static_cast<const uint16_t*>(R), static_cast<uint16_t*>(Z), static_cast<uint16_t*>(Y), join == FPDT_TW_JOIN_TIMES,
                                      all_wide(n_out, {B, R, Z, Y})};
        // (rows that are few for each expert, or weights that are few: us, 8 experts of 4096 x 14336 with a gate, 8 rows 111, tiles 136, 16 rows 152 and 164, 32 rows
        // 164-183 and 159-188, card by card, 64 rows 201 and 196; 64 of 2048 x 1536, 64 rows 53 and 70; 8 of 1024 x 2048, 16 rows 9 and 12)
        if (rows <= FEW_ROWS && (rows <= 4 * experts || few_pays(16, (int64_t)experts * n_in * n_out))) {
            experts_few_kernel<ACT><<<dim3((unsigned)((n_out + FEW_COLS - 1) / FEW_COLS), (unsigned)experts), FEW_WAVES * 64, 0, st>>>(
                static_cast<const uint16_t*>(X), static_cast<const uint16_t*>(W), n_in, n_out, g, behind);
            return;
        }
        by_group_tile(plan, [&](auto wm, auto wn) {
            experts_affine_kernel<ACT, decltype(wm)::value, decltype(wn)::value>
                <<<grid_of(plan.tiles), NTHREAD, 0, st>>>(static_cast<const uint16_t*>(X), static_cast<const uint16_t*>(W), n_in, n_out, g, behind);
        });
    });
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // extern "C"
