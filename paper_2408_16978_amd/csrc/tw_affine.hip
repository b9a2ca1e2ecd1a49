// Products with bias, activation and residual or gate behind them, and the backward of what is behind them (include/fpdt_tokenwise.h:
// fpdt_tw_affine_*).
//
//     z = x W^T + b,   y = act(z) + r  or  act(z) r
//     dz = dy act'(z) (r),   dr = dy act(z),   db += sum_rows dz
//
// The products run the tile loop of tw_gemm_tile.h, which hands finished tiles to an Epilogue.
#include <cmath>
#include <type_traits>

#include "tw_affine.h"
#include "tw_gemm.h"

namespace fpdt_tw {
namespace {

constexpr int64_t MOST_ROWS = (int64_t)1 << 24;  // of one dense product

template <int ACT, int WMT, int WNT>
__global__ __launch_bounds__(NTHREAD, 1) void affine_kernel(Operand A, Operand B, int K, int M, int N, Units u, float* part, Epilogue<ACT> behind)
{
    __shared__ __attribute__((aligned(256))) u32x4 ring[ring_bytes(WMT, WNT) / 16];
    Unit at;
    if (!find_unit(u, at)) return;
    const int unit_stages = at.is_part ? u.split_stages : K / STAGE_K;
    auto part_of = [&](size_t elems) { return part + ((size_t)at.split * (unsigned)(u.tiles - u.whole) + (at.id - (unsigned)u.whole)) * elems; };
    product_tile<false, false, false, false, WMT, WNT>(ring, A, B, K, nullptr, N, M, N, at.tile_m, at.tile_n, (int)at.split * unit_stages, unit_stages, at.is_part, part_of, behind);
}

// The divided tiles of a product, as tw_split_sum_kernel adds them, and what is behind it.
template <int ACT>
__global__ __launch_bounds__(256) void affine_sum_kernel(const float* part, Units u, int first, int tm, int tn, int M, int N, Epilogue<ACT> behind)
{
    const unsigned i = (unsigned)first + blockIdx.y;
    int tile_m, tile_n;
    tile_of((unsigned)u.whole + i, (unsigned)u.tiles / (unsigned)u.tiles_n, (unsigned)u.tiles_n, tile_m, tile_n);
    const int at = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;  // within the tile: tm * tn is a multiple of 1024
    const int m = tile_m * tm + at / tn, n = tile_n * tn + at % tn;
    if (m >= M || n >= N) return;
    const size_t stride = (size_t)(u.tiles - u.whole) * tm * tn;
    const float* p = part + (size_t)i * tm * tn + at;
    floatx4 v = *reinterpret_cast<const floatx4*>(p);
    for (int s = 1; s < u.splits; ++s) v += *reinterpret_cast<const floatx4*>(p + s * stride);
    behind.four(v, m, n, N);
}

template <int ACT, int MT> __global__ __launch_bounds__(FEW_WAVES * 64) void affine_few_kernel(const uint16_t* X, const uint16_t* W, int K, int M, int N, Epilogue<ACT> behind)
{
    __shared__ __attribute__((aligned(16))) float sums[few_lds<MT>];
    few_rows<ACT, MT>(sums, X, W, K, M, N, blockIdx.x * FEW_COLS, behind);
}

// ---- backward of what is behind a product -------------------------------------------------
// dz = dy act'(z) (r), dr = dy act(z); the columns' sums of dz in fp32 before it is rounded.
//
// Bound by the memory, and with GELU nearly by the vector instructions: every tensor is read or written once, eight columns a lane (16384 x 10240, us and TB/s: the sums alone
// 61, 5.5, GELU with them 195, 5.2, SILU and gate 319, 5.3).  A workgroup of `cols` x (256 / cols) threads walks the rows of its
// slice and keeps its columns' sums in registers; where an expert's rows end in the slice they are left as a row of partial sums, number slice + expert
// (no two pairs that meet have the same number), for affine_sums_kernel: no atomics, the same order of sums in every call.
struct Backward {
    const uint16_t *Z, *R, *dY;
    uint16_t *dZ, *dR;
    float* partial;  // or NULL: no sums
    int64_t rows;
    int n, experts, cols;
    const int32_t* offsets;  // or NULL: all rows are one expert's
    int64_t slice;           // rows of a slice
};
__device__ __forceinline__ int64_t start_of(const int32_t* offsets, int e, int64_t rows)
{
    if (!offsets) return e ? rows : 0;
    return offset_of(offsets, e, (int)rows);
}

template <int ACT, bool TIMES, bool WHOLE> __global__ __launch_bounds__(256) void affine_bwd_kernel(Backward b)
{
    constexpr int V = 8, U = 4;
    constexpr bool BEHIND = TIMES || ACT != FPDT_TW_ACT_NONE;
    __shared__ float lds[256 * V];
    const int tc = threadIdx.x % b.cols, tr = threadIdx.x / b.cols, lines = 256 / b.cols, c = ((int)blockIdx.x * b.cols + tc) * V, left = b.n - c;
    const int64_t used = start_of(b.offsets, b.experts, b.rows), begin = start_of(b.offsets, 0, b.rows), from = (int64_t)blockIdx.y * b.slice;
    const int64_t last = from + b.slice < used ? from + b.slice : used;
    int64_t row = from < begin ? begin : from;  // rows in front of the first expert's are nobody's
    int e = 0;
    for (int up = b.experts; up - e > 1;) {  // the last expert that begins at or before this row
        const int mid = (e + up) / 2;
        if (start_of(b.offsets, mid, b.rows) <= row) e = mid;
        else up = mid;
    }
    auto fetch = [&](const uint16_t* p, int64_t at) {
        if (WHOLE || left >= V) return load_once<V>(p + at);
        Vec<uint16_t, V> v;
#pragma unroll
        for (int i = 0; i < V; ++i) v.e[i] = i < left ? p[at + i] : 0;
        return v;
    };
    auto put = [&](uint16_t* p, int64_t at, const Vec<uint16_t, V>& v) {
        if (WHOLE || left >= V) {
            store_once(p + at, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) p[at + i] = v.e[i];
        }
    };
    while (row < last) {
        while (e + 1 < b.experts && start_of(b.offsets, e + 1, b.rows) <= row) ++e;  // experts without rows
        int64_t end = start_of(b.offsets, e + 1, b.rows);
        end = end > row && end < last ? end : last;
        float sum[V] = {};
        // n rows from r on, `lines` apart: all of them are requested first, and nothing is conditional, so that no wait for them is one for the rows stored before
        auto rows = [&](int64_t r, auto n_tag) __attribute__((always_inline)) {
            constexpr int n = decltype(n_tag)::value;
            const int64_t at0 = r * b.n + c, step = (int64_t)lines * b.n;
            Vec<uint16_t, V> dy[n], z[n], gate[n];
#pragma unroll
            for (int k = 0; k < n; ++k) {
                dy[k] = fetch(b.dY, at0 + k * step);
                if (BEHIND) z[k] = fetch(b.Z, at0 + k * step);
                if (TIMES) gate[k] = fetch(b.R, at0 + k * step);
            }
#pragma unroll
            for (int k = 0; k < n; ++k) {
                float dz[V], dr[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float g = to_float(dy[k].e[i]);
                    dz[i] = g;
                    if (BEHIND) {
                        float y;
                        dz[i] *= slope_of<ACT>(to_float(z[k].e[i]), y);
                        if (TIMES) dz[i] *= to_float(gate[k].e[i]), dr[i] = g * y;
                    }
                    sum[i] += dz[i];
                }
                if (BEHIND || b.dZ) put(b.dZ, at0 + k * step, rounded<V>(dz, uint16_t()));
                if (TIMES && b.dR) put(b.dR, at0 + k * step, rounded<V>(dr, uint16_t()));
            }
        };
        if (left > 0) {
            int64_t r = row + tr;
            for (; r + (U - 1) * lines < end; r += U * lines) rows(r, Int<U>());
            for (; r < end; r += lines) rows(r, Int<1>());
        }
        if (b.partial) {
            float* out = b.partial + ((int64_t)blockIdx.y + e) * b.n;
#pragma unroll
            for (int i = 0; i < V; ++i) lds[threadIdx.x * V + i] = sum[i];
            __syncthreads();
            for (int i = threadIdx.x; i < b.cols * V; i += 256) {
                float v = 0.f;
                for (int k = 0; k < lines; ++k) v += lds[k * b.cols * V + i];
                const int col = (int)blockIdx.x * b.cols * V + i;
                if (col < b.n) out[col] = v;
            }
            __syncthreads();
        }
        row = end;
    }
}

// dB of expert blockIdx.y += its partial sums, in 64 bits: rounded once, with what was there.  32 columns and 32 shares of the sums a workgroup.
__global__ __launch_bounds__(1024) void affine_sums_kernel(Backward b, float* dB)
{
    constexpr int COLS = 32, SHARES = 1024 / COLS, U = 8;
    __shared__ double part[SHARES][COLS];
    const int lane = threadIdx.x % COLS, w = threadIdx.x / COLS, c = blockIdx.x * COLS + lane, e = blockIdx.y;
    const int64_t begin = start_of(b.offsets, e, b.rows), end = start_of(b.offsets, e + 1, b.rows);
    if (end <= begin) return;
    const int64_t first = begin / b.slice + e, n = (end - 1) / b.slice + e - first + 1;
    const float* p = b.partial + first * b.n + c;
    double v = 0;
    if (c < b.n) {
        int64_t r = w;
        for (; r + (U - 1) * SHARES < n; r += U * SHARES) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = p[(r + u * SHARES) * b.n];
#pragma unroll
            for (int u = 0; u < U; ++u) v += x[u];
        }
        for (; r < n; r += SHARES) v += p[r * b.n];
    }
    part[w][lane] = v;
    __syncthreads();
    if (w || c >= b.n) return;
#pragma unroll
    for (int i = 1; i < SHARES; ++i) v += part[i][lane];
    float* d = dB + (int64_t)e * b.n + c;
    *d = (float)(*d + v);
}

// ---- host side ----------------------------------------------------------------------------
size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// The dense product: its copies and partial sums in the workspace.  Copies are made where rows are no multiple of 16 bytes, of X for
// PIECE rows at a time.
constexpr int64_t PIECE = 32768;
int pitch_of(int n) { return n <= 64 ? (n + 7) / 8 * 8 : (n + 63) / 64 * 64; }
struct Layout {
    int64_t piece;       // rows of a product
    size_t w, x, parts;  // bytes
};
size_t parts_of(const Plan& p) { return p.u.splits > 1 ? (size_t)p.u.splits * (p.u.tiles - p.u.whole) * (64 * p.wmt) * (64 * p.wnt) * 4 : 0; }
Plan plan_of(int64_t rows, int n_in, int n_out) { return plan_launch(rows, n_out, (n_in < SK ? SK : n_in) / SK); }
Layout layout_of(int64_t rows, int n_in, int n_out)
{
    Layout l = {};
    const bool copy = n_in % 8 != 0;
    l.piece = copy ? PIECE : MOST_ROWS;
    if (copy) l.w = al256((size_t)n_out * pitch_of(n_in) * 2), l.x = al256((size_t)(rows < PIECE ? rows : PIECE) * pitch_of(n_in) * 2);
    for (int64_t n : {rows < l.piece ? rows : l.piece, rows % l.piece})
        if (n > 0) {
            const size_t b = al256(parts_of(plan_of(n, n_in, n_out)));
            if (b > l.parts) l.parts = b;
        }
    return l;
}

// Threads along the columns: the most of which at most a ninth are idle, or those of which the fewest are (30001 rows of 2560 columns, SILU: 256 threads, a quarter
// of the second 256 at work, 104 us, 64 87; 100000 rows of 264 columns: 8 threads 76 us, 64 40).
int lanes_of(int n)
{
    const int accesses = (n + 7) / 8;
    int best = 8, least = 1 << 30;
    while (best < 32 && best < accesses) best *= 2;
    if (accesses < 32) return best;
    for (int cols = 256; cols >= 32; cols /= 2) {
        const int threads = (accesses + cols - 1) / cols * cols;
        if (threads * 8 <= accesses * 9) return cols;
        if (threads < least) best = cols, least = threads;
    }
    return best;
}
// Rows of a slice: 1536 workgroups where there are rows enough, so that partial sums stay a small part of the tensors, and two rows a thread at
// least (16384 rows of 10240 columns, GELU, us: 1024 workgroups 212, 1536 200, 2048 204).
int64_t slice_of(int64_t rows, int n)
{
    const int cols = lanes_of(n), wide = (n + cols * 8 - 1) / (cols * 8), lines = 256 / cols;
    const int64_t most = wide < 1536 ? 1536 / wide : 1, least = 2 * lines, slice = (rows + most - 1) / most;
    return slice > least ? (slice + lines - 1) / lines * lines : least;
}

}  // namespace
}  // namespace fpdt_tw

using namespace fpdt_tw;

extern "C" {

size_t fpdt_tw_affine_workspace_bytes(int64_t rows, int n_in, int n_out)
{
    if (rows <= 0 || n_in <= 0 || n_out <= 0 || n_in > MOST_WIDTH || n_out > MOST_WIDTH || rows > INT32_MAX) return 0;
    const Layout l = layout_of(rows, n_in, n_out);
    return l.w + l.x + l.parts + 256;  // (never 0 for what is valid)
}

int fpdt_tw_affine_fwd(const void* X, const void* W, const void* B, const void* R, void* Z, void* Y, int64_t rows, int n_in, int n_out, int act, int join,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    if (!X || !W || !Y) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_sizes(rows, n_in, n_out);
    if (rc != TW_OK || (rc = check_kind(act, join)) != TW_OK) return rc;
    if (join == FPDT_TW_JOIN_TIMES && !R) return fail(TW_INVALID, "JOIN_TIMES needs R");
    for (const void* p : {X, W, B, R, (const void*)Z, (const void*)Y})
        if (misaligned(p, 2)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    if (n_in % 8 == 0 && (misaligned(X, 16) || misaligned(W, 16))) return fail(TW_INVALID, "X and W must be 16-byte aligned where n_in is a multiple of 8");
    const size_t need = fpdt_tw_affine_workspace_bytes(rows, n_in, n_out);
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256))
        return fail(TW_WORKSPACE, "workspace NULL, misaligned or too small (%zu < %zu bytes)", workspace_bytes, need);
    const size_t out = (size_t)rows * n_out * 2;
    const Arg args[] = {{"X", X, (size_t)rows * n_in * 2, false}, {"W", W, (size_t)n_in * n_out * 2, false}, {"B", B, (size_t)n_out * 2, false}, {"R", R, out, false},
                        {"Z", Z, out, true}, {"Y", Y, out, true}, {"the workspace", workspace, need, true}};
    const int same[][2] = {{3, 5}};
    if ((rc = check_apart(args, 7, same, 1)) != TW_OK) return rc;

    hipStream_t st = static_cast<hipStream_t>(stream);
    const Layout l = layout_of(rows, n_in, n_out);
    char* ws = static_cast<char*>(workspace);
    float* part = reinterpret_cast<float*>(ws + l.w + l.x);
    Operand w = {static_cast<const uint16_t*>(W), n_in, n_out};
    if (l.w) {
        w.p = reinterpret_cast<const uint16_t*>(ws), w.ld = pitch_of(n_in);
        realign(W, n_out, n_in, n_in, ws, w.ld, st);
    }
    const bool wide = all_wide(n_out, {B, R, Z, Y});
    const int tall = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    if (rows <= FEW_ROWS && n_in % 8 == 0 && few_pays(rows, (int64_t)n_in * n_out)) {
        by_act(act, [&](auto a) {
            constexpr int ACT = decltype(a)::value;
            const Epilogue<ACT> behind = {static_cast<const uint16_t*>(B), static_cast<const uint16_t*>(R), static_cast<uint16_t*>(Z), static_cast<uint16_t*>(Y),
                                          join == FPDT_TW_JOIN_TIMES, wide};
            const auto kernel = tall == 1 ? affine_few_kernel<ACT, 1> : tall == 2 ? affine_few_kernel<ACT, 2> : affine_few_kernel<ACT, 4>;
            kernel<<<(unsigned)((n_out + FEW_COLS - 1) / FEW_COLS), FEW_WAVES * 64, 0, st>>>(static_cast<const uint16_t*>(X), w.p, n_in, (int)rows, n_out, behind);
        });
        HIP_TRY(hipGetLastError());
        return TW_OK;
    }
    for (int64_t r0 = 0; r0 < rows; r0 += l.piece) {
        const int m = (int)(rows - r0 < l.piece ? rows - r0 : l.piece);
        const Plan plan = plan_of(m, n_in, n_out);
        if (plan.u.tiles == 0) return fail(TW_UNSUPPORTED, "product beyond the launch limits");
        Operand x = {static_cast<const uint16_t*>(X) + r0 * n_in, n_in, m};
        if (l.x) {
            realign(x.p, m, n_in, n_in, ws + l.w, w.ld, st);
            x.p = reinterpret_cast<const uint16_t*>(ws + l.w), x.ld = w.ld;
        }
        const int64_t at = r0 * n_out;
        const int64_t divided = plan.u.tiles - plan.u.whole, parts = divided * plan.u.splits;
        const unsigned grid = 8 * ((unsigned)((plan.u.whole + 7) / 8) + (unsigned)((parts + 7) / 8));
        by_act(act, [&](auto a) {
            constexpr int ACT = decltype(a)::value;
            const Epilogue<ACT> behind = {static_cast<const uint16_t*>(B), R ? static_cast<const uint16_t*>(R) + at : nullptr, Z ? static_cast<uint16_t*>(Z) + at : nullptr,
                                          static_cast<uint16_t*>(Y) + at, join == FPDT_TW_JOIN_TIMES, wide};
            by_tile(plan.wmt, plan.wnt, [&](auto wm, auto wn) {
                affine_kernel<ACT, decltype(wm)::value, decltype(wn)::value><<<grid, NTHREAD, 0, st>>>(x, w, n_in, m, n_out, plan.u, part, behind);
            });
            const int tm = 64 * plan.wmt, tn = 64 * plan.wnt;
            for (int64_t t0 = 0; plan.u.splits > 1 && t0 < divided; t0 += 65535)
                affine_sum_kernel<ACT><<<dim3(tm * tn / 1024, (unsigned)(divided - t0 < 65535 ? divided - t0 : 65535)), 256, 0, st>>>(part, plan.u, (int)t0, tm, tn, m,
                                                                                                                                      n_out, behind);
        });
    }
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

size_t fpdt_tw_affine_bwd_workspace_bytes(int64_t rows, int n_out, int experts)
{
    if (rows <= 0 || n_out <= 0 || experts <= 0 || n_out > MOST_WIDTH || rows > INT32_MAX || experts > MOST_EXPERTS) return 0;
    const int64_t slice = slice_of(rows, n_out);
    return al256((size_t)((rows + slice - 1) / slice + experts) * n_out * 4);
}

int fpdt_tw_affine_bwd(const void* Z, const void* R, const void* dY, void* dZ, void* dR, float* dB, int64_t rows, int n_out, int act, int join,
                       const int32_t* offsets, int experts, void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    if (!dY) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_sizes(rows, 1, n_out);
    if (rc != TW_OK || (rc = check_kind(act, join)) != TW_OK) return rc;
    if (experts <= 0 || (!offsets && experts != 1)) return fail(TW_INVALID, "experts must be positive, and 1 without offsets");
    if (experts > MOST_EXPERTS) return fail(TW_UNSUPPORTED, "experts=%d beyond %d", experts, MOST_EXPERTS);
    const bool times = join == FPDT_TW_JOIN_TIMES, behind = times || act != FPDT_TW_ACT_NONE;
    if (behind && (!Z || !dZ)) return fail(TW_INVALID, "an activation's or gate's backward needs Z and dZ");
    if (times && !R) return fail(TW_INVALID, "JOIN_TIMES needs R");
    if (!times && dR) return fail(TW_INVALID, "the gradient of an R that is added is dY: dR must be NULL");
    if (!dZ && !dB) return fail(TW_INVALID, "nothing to compute: dZ and dB are NULL");
    for (const void* p : {Z, R, dY, (const void*)dZ, (const void*)dR})
        if (misaligned(p, 2)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    if (misaligned(dB, 4) || misaligned(offsets, 4)) return fail(TW_INVALID, "dB or offsets is not aligned to its elements");
    const size_t need = dB ? fpdt_tw_affine_bwd_workspace_bytes(rows, n_out, experts) : 0, n = (size_t)rows * n_out * 2;
    if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 256)))
        return fail(TW_WORKSPACE, "workspace NULL, misaligned or too small (%zu < %zu bytes)", workspace_bytes, need);
    const Arg args[] = {{"Z", Z, n, false}, {"R", R, n, false}, {"dY", dY, n, false}, {"dZ", dZ, n, true}, {"dR", dR, n, true}, {"dB", dB, (size_t)experts * n_out * 4, true},
                        {"offsets", offsets, (size_t)(experts + 1) * 4, false}, {"the workspace", need ? workspace : nullptr, need, true}};
    const int same[][2] = {{0, 3}, {1, 3}, {2, 3}, {0, 4}, {1, 4}, {2, 4}};
    if ((rc = check_apart(args, 8, same, 6)) != TW_OK) return rc;

    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t slice = slice_of(rows, n_out), slices = (rows + slice - 1) / slice;
    Backward b = {static_cast<const uint16_t*>(Z), static_cast<const uint16_t*>(R), static_cast<const uint16_t*>(dY), static_cast<uint16_t*>(dZ), static_cast<uint16_t*>(dR),
                  dB ? static_cast<float*>(workspace) : nullptr, rows, n_out, experts, lanes_of(n_out), offsets, slice};
    const dim3 grid((unsigned)((n_out + b.cols * 8 - 1) / (b.cols * 8)), (unsigned)slices);
    by_act(act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        auto run = [&](auto t, auto w) { affine_bwd_kernel<ACT, decltype(t)::value, decltype(w)::value><<<grid, 256, 0, st>>>(b); };
        typedef std::true_type Yes;
        typedef std::false_type No;
        if (times && n_out % 8 == 0) run(Yes(), Yes());
        else if (times) run(Yes(), No());
        else if (n_out % 8 == 0) run(No(), Yes());
        else run(No(), No());
    });
    if (dB) affine_sums_kernel<<<dim3((unsigned)((n_out + 31) / 32), (unsigned)experts), 1024, 0, st>>>(b, dB);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // extern "C"
