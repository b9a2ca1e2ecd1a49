// Dense bf16 products of the token-wise chunked operations (Sec. 4.1, 5.4: the per-chunk QKV
// projection, the feed-forward block and the output projection of the loss are plain GEMMs over
// one chunk of tokens at a time) on v_mfma_f32_16x16x32_bf16: stages of 64 k in LDS, filled by direct
// global -> LDS copies two stages ahead, four waves (one per SIMD) per output tile of up to
// 256 x 256.
//
//   C[M,N] (+)= sum_k Aop[m,k] * Bop[n,k]          fp32 accumulation, C bf16 or fp32
//
// Every product of the library is of this form once each operand is read either as stored
// (row = row, k = column) or transposed (row = column, k = row).  Both are read in place: the copy
// engine fetches 16-byte pieces of the stored rows, a plain LDS read delivers the fragments of the
// first form and a transposing LDS read those of the second.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>
#include <type_traits>
#include <utility>
#include <vector>

#include "tw_gemm.h"
#include "tw_gemm_tile.h"

namespace fpdt_tw {

namespace {

// ---- realign ----------------------------------------------------------------------------
// The product kernel copies 16-byte pieces of its operands' rows.  An operand that does not offer that (a
// width that is not a multiple of 8, a base that is not 16-byte aligned), or that the product overwrites, is
// copied once: X [R, C] with its columns rounded up to 8, zero behind C, rows `pitch` elements apart.
__global__ __launch_bounds__(256) void tw_realign_kernel(const uint16_t* __restrict__ X, int64_t R, int64_t C, int64_t ld,
                                                         u32x4* __restrict__ out, int64_t pitch)
{
    const int64_t pieces = (C + 7) / 8, n = R * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = n >> 32 ? i / pieces : (unsigned)i / (unsigned)pieces, c = (i - r * pieces) * 8;
        u32x4 v;
        if (c + 8 <= C) {  // (16 bytes at any even address in one access)
            __builtin_memcpy(&v, X + r * ld + c, 16);
        } else {
            unsigned e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = c + j < C ? X[r * ld + c + j] : 0u;
            v = u32x4{e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16), e[6] | (e[7] << 16)};
        }
        out[r * (pitch / 8) + c / 8] = v;
    }
}

// ---- product ----------------------------------------------------------------------------
template <bool TA, bool TB, bool OUT_F32, bool ACCUM, int WMT, int WNT>
__global__ __launch_bounds__(NTHREAD, 1) void tw_gemm_kernel(Operand A, Operand B, int K, void* __restrict__ Cout, int64_t ldc,
                                                              int M, int N, Units u, float* __restrict__ part)
{
    __shared__ __attribute__((aligned(256))) u32x4 ring[ring_bytes(WMT, WNT) / 16];
    Unit at;
    if (__builtin_expect(find_unit(u, at), 1)) {
        const int unit_stages = at.is_part ? u.split_stages : K / STAGE_K;
        auto part_of = [&](size_t elems) { return part + ((size_t)at.split * (unsigned)(u.tiles - u.whole) + (at.id - (unsigned)u.whole)) * elems; };
        product_tile<TA, TB, OUT_F32, ACCUM, WMT, WNT>(ring, A, B, K, Cout, ldc, M, N, at.tile_m, at.tile_n, (int)at.split * unit_stages, unit_stages, at.is_part, part_of,
                                                       Nothing());
    }
}

// The divided tiles of a product: C (+)= the sums of their splits, part [split][tile][TM x TN] fp32.
// Memory-bound: (splits + 1) passes over those tiles.
template <bool OUT_F32, bool ACCUM>
__global__ __launch_bounds__(256) void tw_split_sum_kernel(const float* __restrict__ part, Units u, int first, int tm, int tn, void* __restrict__ Cout,
                                                            int64_t ldc, int M, int N)
{
    typedef typename std::conditional<OUT_F32, float, uint16_t>::type out_t;
    typedef out_t out4 __attribute__((ext_vector_type(4)));
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
    out_t* c = static_cast<out_t*>(Cout) + (size_t)m * ldc + n;
    if (n + 4 <= N && ldc % 4 == 0 && reinterpret_cast<uintptr_t>(Cout) % (4 * sizeof(out_t)) == 0) {
        out4 o = {};
        if (ACCUM) o = *reinterpret_cast<const out4*>(c);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = combine<ACCUM>(v[r], o[r]);
        *reinterpret_cast<out4*>(c) = o;
    } else {
        for (int r = 0; r < 4 && n + r < N; ++r) c[r] = combine<ACCUM>(v[r], ACCUM ? c[r] : out_t(0));
    }
}

// ---- host side: scratch and the per-call cache of realigned weights --------------
struct Pool {
    char* base = nullptr;
    size_t cap = 0, off = 0;
    std::vector<void*> retired;  // outgrown buffers: work already enqueued may still read them
};
struct Realigned {
    const void* src;
    int64_t R, C, ld;
    const uint16_t* copy;
};
Pool g_pool[64];
std::vector<Realigned> g_cache;  // weights realigned during the current library call
std::mutex g_mu;

int pool_take(Pool& p, size_t bytes, char** out)
{
    bytes = (bytes + 255) & ~(size_t)255;
    if (p.off + bytes > p.cap) {
        // Grow: a new buffer; the old one stays alive (kernels in flight, and the rest of this call, read
        // it) until exit.  The call's offsets go on as if all of it were in the new buffer, so that it
        // holds all of the next call of these sizes, which may be captured.
        size_t want = p.cap ? p.cap * 2 : (size_t)256 << 20;
        while (want < p.off + bytes) want *= 2;
        void* nb = nullptr;
        if (hipMalloc(&nb, want) != hipSuccess) {
            (void)hipGetLastError();
            return 1;
        }
        if (p.base) p.retired.push_back(p.base);
        p.base = static_cast<char*>(nb);
        p.cap = want;
    }
    *out = p.base + p.off;
    p.off += bytes;
    return 0;
}

// A lane's offset within its tile (255 rows of form N, 7 of form T) is kept in 32 bits
constexpr int64_t MAX_PITCH = (int64_t)1 << 23;    // elements between rows along k
constexpr int64_t MAX_PITCH_T = (int64_t)1 << 28;  // and between the rows of k, form T
constexpr int64_t COPY_PAD = 64;                   // a copy's rows are this many elements further apart at most

// The bytes that a product writes
struct Written {
    const void* C;
    int64_t rows, cols, ld;
    int size;
    bool overlaps(const void* X, int64_t R, int64_t cols_x, int64_t ld_x) const
    {
        const uintptr_t c = reinterpret_cast<uintptr_t>(C), x = reinterpret_cast<uintptr_t>(X);
        return x < c + (uintptr_t)((rows - 1) * ld + cols) * size && c < x + (uintptr_t)((R - 1) * ld_x + cols_x) * 2;
    }
};

// Can the product kernel read X [R, C] where it is?
bool readable(const void* X, int64_t R, int64_t C, int64_t ld, bool k_rows, bool padded, const Written& out)
{
    return (C % 8 == 0 || padded) && ld % 8 == 0 && ld < (k_rows ? MAX_PITCH_T : MAX_PITCH) &&
           reinterpret_cast<uintptr_t>(X) % 16 == 0 && !out.overlaps(X, R, C, ld);
}

// X [R, C], leading dimension ld, as the product kernel can read it: in place, or copied.  `k_rows`: the
// contraction runs over the rows of X.  `padded`: rows are followed by zeros up to a multiple of 8.
// An operand that the product itself overwrites (Y in the place of X) is copied: tiles are stored while
// others still read their rows.
int take_operand(Pool& pool, const void* X, int64_t R, int64_t C, int64_t ld, bool k_rows, bool padded, bool cache, const Written& out,
                 hipStream_t st, Operand* res)
{
    res->rows = (int)(k_rows ? (C + 7) / 8 * 8 : R);
    if (readable(X, R, C, ld, k_rows, padded, out)) {
        res->p = static_cast<const uint16_t*>(X);
        res->ld = ld;
    } else {
        const int64_t C2 = (C + 7) / 8 * 8;
        // whole cache lines from row to row: a stage's part of a row is a line (form N: 64 k, form T: 64 columns), and with
        // 8208 bytes from row to row in place of 8320 it lay in two (Y of 16384 x 4097 x 4096: 493 -> 451 us, in 8 chunks
        // 626 -> 542)
        res->ld = C2 <= 64 ? C2 : (C2 + 63) / 64 * 64;
        res->p = nullptr;
        if (cache)
            for (const Realigned& c : g_cache)
                if (c.src == X && c.R == R && c.C == C && c.ld == ld) res->p = c.copy;
        if (!res->p) {
            char* mem = nullptr;
            if (pool_take(pool, (size_t)R * res->ld * 2, &mem)) return 1;
            realign(X, R, C, ld, mem, res->ld, st);
            res->p = reinterpret_cast<const uint16_t*>(mem);
            if (cache) g_cache.push_back({X, R, C, ld, res->p});
        }
    }
    return res->ld >= (k_rows ? MAX_PITCH_T : MAX_PITCH) ? 2 : 0;
}

}  // namespace

void realign(const void* X, int64_t R, int64_t C, int64_t ld, void* out, int64_t pitch, hipStream_t st)
{
    const int64_t blocks = (R * ((C + 7) / 8) + 255) / 256;
    tw_realign_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), 256, 0, st>>>(static_cast<const uint16_t*>(X), R, C, ld, static_cast<u32x4*>(out), pitch);
}

void begin_call()
{
    std::lock_guard<std::mutex> lk(g_mu);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return;
    g_cache.clear();
    g_pool[dev].off = 0;  // everything enqueued earlier on the stream is ordered before what follows
}

bool reads_in_place(const void* A, int64_t rows, int64_t k, const void* C, int64_t cols)
{
    return readable(A, rows, k, k, false, false, Written{C, rows, cols, cols, 2});
}

void* scratch(size_t bytes)
{
    std::lock_guard<std::mutex> lk(g_mu);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return nullptr;
    char* mem = nullptr;
    return pool_take(g_pool[dev], bytes, &mem) ? nullptr : mem;
}

// The launch of a product (or, with u.whole = 0 and one split at a time, of one k segment of it)
static int launch_product(const Plan& plan, int a_transposed, int b_transposed, const Operand& a, const Operand& b, int M, int N, int K,
                          void* C, int64_t ldc, bool c_f32, bool accumulate, float* part, hipStream_t st)
{
    const Units& u = plan.u;
    const int64_t parts = (int64_t)(u.tiles - u.whole) * u.splits;
    const unsigned grid = 8 * ((unsigned)((u.whole + 7) / 8) + (unsigned)((parts + 7) / 8));
#define TW_LAUNCH_TILE(TA, TB, F32, ACC, WM, WN) tw_gemm_kernel<TA, TB, F32, ACC, WM, WN><<<grid, NTHREAD, 0, st>>>(a, b, K, C, ldc, M, N, u, part)
#define TW_LAUNCH(TA, TB, F32, ACC)                                             \
    do {                                                                        \
        if (plan.wnt == 2) TW_LAUNCH_TILE(TA, TB, F32, ACC, 2, 2);              \
        else if (plan.wmt == 4) TW_LAUNCH_TILE(TA, TB, F32, ACC, 4, 4);         \
        else if (plan.wmt == 3) TW_LAUNCH_TILE(TA, TB, F32, ACC, 3, 4);         \
        else if (plan.wmt == 2) TW_LAUNCH_TILE(TA, TB, F32, ACC, 2, 4);         \
        else TW_LAUNCH_TILE(TA, TB, F32, ACC, 1, 4);                            \
    } while (0)
    // the forms and outputs that the library's operations use
    if (!a_transposed && !b_transposed && !accumulate) {
        if (c_f32) TW_LAUNCH(false, false, true, false);
        else TW_LAUNCH(false, false, false, false);
    } else if (!a_transposed && b_transposed && !c_f32) {
        if (accumulate) TW_LAUNCH(false, true, false, true);
        else TW_LAUNCH(false, true, false, false);
    } else if (a_transposed && b_transposed && c_f32 && accumulate) {
        TW_LAUNCH(true, true, true, true);
    } else {
        return 2;
    }
#undef TW_LAUNCH
#undef TW_LAUNCH_TILE
    return 0;
}

static size_t part_bytes(const Plan& plan) { return (size_t)plan.u.splits * (plan.u.tiles - plan.u.whole) * (64 * plan.wmt) * (64 * plan.wnt) * 4; }

static void launch_split_sum(const Plan& plan, const float* part, int M, int N, void* C, int64_t ldc, bool c_f32, bool accumulate, hipStream_t st)
{
    const int tm = 64 * plan.wmt, tn = 64 * plan.wnt, divided = plan.u.tiles - plan.u.whole;
    for (int t0 = 0; t0 < divided; t0 += 65535) {  // the grid's second dimension
        const Units& u = plan.u;
        const dim3 grid((unsigned)(tm * tn / 1024), (unsigned)(divided - t0 < 65535 ? divided - t0 : 65535));
        if (c_f32 && accumulate) tw_split_sum_kernel<true, true><<<grid, 256, 0, st>>>(part, u, t0, tm, tn, C, ldc, M, N);
        else if (c_f32) tw_split_sum_kernel<true, false><<<grid, 256, 0, st>>>(part, u, t0, tm, tn, C, ldc, M, N);
        else if (accumulate) tw_split_sum_kernel<false, true><<<grid, 256, 0, st>>>(part, u, t0, tm, tn, C, ldc, M, N);
        else tw_split_sum_kernel<false, false><<<grid, 256, 0, st>>>(part, u, t0, tm, tn, C, ldc, M, N);
    }
}

static int product(Pool& pool, int a_transposed, int b_transposed, int M, int N, int K, const void* A, int64_t lda, const void* B,
                   int64_t ldb, void* C, int64_t ldc, bool c_f32, bool accumulate, bool cache_b, hipStream_t st)
{
    const size_t off0 = pool.off;
    const Plan plan = plan_launch(M, N, (K < SK ? SK : K) / SK);
    if (plan.u.tiles == 0) return 2;
    // Aop[m,k]: A stored [M,K] (as is) or [K,M] (transposed); Bop[n,k]: B stored [N,K] or [K,N]
    const Written out = {C, M, N, ldc, c_f32 ? 4 : 2};
    Operand pa, pb;
    int rc = take_operand(pool, B, b_transposed ? K : N, b_transposed ? N : K, ldb, b_transposed, false, cache_b, out, st, &pb);
    if (rc) return rc;
    const size_t mark = pool.off;  // what follows is scratch of this product only
    rc = take_operand(pool, A, a_transposed ? K : M, a_transposed ? M : K, lda, a_transposed, lda > (a_transposed ? M : K), false, out, st, &pa);
    if (rc) return rc;
    float* part = nullptr;
    if (plan.u.splits > 1) {
        char* mem = nullptr;
        if (pool_take(pool, part_bytes(plan), &mem)) return 1;
        part = reinterpret_cast<float*>(mem);
    }
    rc = launch_product(plan, a_transposed, b_transposed, pa, pb, M, N, K, C, ldc, c_f32, accumulate, part, st);
    if (rc) return rc;
    if (plan.u.splits > 1) launch_split_sum(plan, part, M, N, C, ldc, c_f32, accumulate, st);
    // The next product's copies run after this launch on the same stream, so this product's scratch
    // is free again: everything it took, or everything behind a weight that stays cached.
    pool.off = cache_b ? mark : off0;
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

static int any_product(Pool& pool, int a_transposed, int b_transposed, int M, int N, int K, const void* A, int64_t lda, const void* B,
                       int64_t ldb, void* C, int64_t ldc, bool c_f32, bool accumulate, bool cache_b, hipStream_t st)
{
    // Rows of k too far apart (form T, an operand of more than 2^28 columns): the columns, which are rows or
    // columns of C, in segments, whose copies have a shorter pitch.  More than 2^30 columns of C in segments
    // too: the last tile would reach behind 2^31.
    constexpr int SEG_T = 1 << 24, SEG_N = 1 << 30;
    const int seg_n = b_transposed && ldb > MAX_PITCH_T - COPY_PAD ? SEG_T : SEG_N;
    if (N > seg_n) {
        for (int64_t n0 = 0; n0 < N; n0 += seg_n) {
            const int rc = any_product(pool, a_transposed, b_transposed, M, (int)(N - n0 < seg_n ? N - n0 : seg_n), K, A, lda,
                                       static_cast<const uint16_t*>(B) + (b_transposed ? n0 : n0 * ldb), ldb,
                                       static_cast<char*>(C) + n0 * (c_f32 ? 4 : 2), ldc, c_f32, accumulate, false, st);
            if (rc) return rc;
        }
        return 0;
    }
    if (a_transposed && lda > MAX_PITCH_T - COPY_PAD && M > SEG_T) {
        for (int64_t m0 = 0; m0 < M; m0 += SEG_T) {
            const int rc = any_product(pool, a_transposed, b_transposed, (int)(M - m0 < SEG_T ? M - m0 : SEG_T), N, K, static_cast<const uint16_t*>(A) + m0, lda, B, ldb,
                                       static_cast<char*>(C) + (size_t)m0 * ldc * (c_f32 ? 4 : 2), ldc, c_f32, accumulate, cache_b, st);
            if (rc) return rc;
        }
        return 0;
    }
    const bool long_a = !a_transposed && lda > MAX_PITCH - COPY_PAD, long_b = !b_transposed && ldb > MAX_PITCH - COPY_PAD;
    if (!long_a && !long_b)
        return product(pool, a_transposed, b_transposed, M, N, K, A, lda, B, ldb, C, ldc, c_f32, accumulate, cache_b, st);
    // Rows too long for the kernel's offsets: k in segments, which are the splits of every tile, one launch
    // each; the long operand's segment is copied out in front of it.
    constexpr int64_t SEG = (int64_t)1 << 22;
    Plan plan = {4, 4, {}};
    const int64_t tiles_n = ((int64_t)N + 255) / 256, tiles = ((int64_t)M + 255) / 256 * tiles_n;
    if (tiles > (int64_t)1 << 30) return 2;
    plan.u = {(int)tiles, (int)tiles_n, 0, (int)((K + SEG - 1) / SEG), 0};
    const size_t off0 = pool.off;
    char* mem = nullptr;
    if (pool_take(pool, part_bytes(plan), &mem)) return 1;
    float* part = reinterpret_cast<float*>(mem);
    for (int i = 0; i < plan.u.splits; ++i) {
        const int64_t k0 = i * SEG, k = K - k0 < SEG ? K - k0 : SEG;
        const size_t off1 = pool.off;
        Operand a, b;
        // (a segment of a long row is never read in place: its pitch is the row's; C is written behind all of them)
        const Written out = {part, 1, 1, 1, 4};
        int rc = take_operand(pool, static_cast<const uint16_t*>(B) + (b_transposed ? k0 * ldb : k0), b_transposed ? k : N, b_transposed ? N : k, ldb, b_transposed, false, false, out, st, &b);
        if (!rc) rc = take_operand(pool, static_cast<const uint16_t*>(A) + (a_transposed ? k0 * lda : k0), a_transposed ? k : M, a_transposed ? M : k, lda, a_transposed, false, false, out, st, &a);
        if (rc) return rc;
        Plan one = plan;
        one.u.splits = 1;
        one.u.split_stages = (int)(k / STAGE_K);
        rc = launch_product(one, a_transposed, b_transposed, a, b, M, N, (int)k, C, ldc, c_f32, accumulate, part + (size_t)i * (part_bytes(one) / 4), st);
        if (rc) return rc;
        pool.off = off1;
    }
    launch_split_sum(plan, part, M, N, C, ldc, c_f32, accumulate, st);
    pool.off = off0;
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

int gemm(int a_transposed, int b_transposed, int M, int N, int K, const void* A, int64_t lda, const void* B,
         int64_t ldb, void* C, int64_t ldc, bool c_f32, bool accumulate, bool cache_b, hipStream_t st)
{
    std::lock_guard<std::mutex> lk(g_mu);
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 1;
    if (M <= 0 || N <= 0 || K <= 0) return 2;
    return any_product(g_pool[dev], a_transposed, b_transposed, M, N, K, A, lda, B, ldb, C, ldc, c_f32, accumulate, cache_b, st);
}

}  // namespace fpdt_tw
