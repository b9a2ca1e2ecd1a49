// Tokens to their experts and back (include/fpdt_tokenwise.h: fpdt_tw_experts_sort, _gather_*, _combine_*).
//
//     place(t, j) = offsets[e] + number of assignments to e = expert(t, j) before (t, j)
//     xs[place(t, j)] = x[t],                  dx[t] = sum_j dxs[place(t, j)] + r[t]
//     y[t] = sum_j w(t, j) ys[place(t, j)] + r[t],   dys[place(t, j)] = w(t, j) dy[t],   dw(t, j) = dy[t] . ys[place(t, j)]
//
// Bound by the memory, but for the sort, which is bound by its launches: a row is read once and written to all its places, or read from all of
// them and written once.
#include <type_traits>

#include "../../include/fpdt_tokenwise.h"
#include "tw_common.h"

namespace {

using namespace fpdt_tw;

constexpr int MOST_EXPERTS = 1024;

// ---- sort -----------------------------------------------------------------------------------
// By counting, and stable, so that a place depends on the choices alone.  A workgroup takes a tile of 1024 `rounds` neighbouring assignments, a wave 64
// `rounds` of them, 64 at a time.  Several tiles: sort_count_kernel counts each tile's assignments to each expert, and every workgroup of
// sort_place_kernel adds up the counts of all tiles and of those before its own: two launches, whose count is what a small sort costs (65536 assignments to 8 experts
// 4.8 and 4.8 us; 32 in one launch 2.8).
constexpr int THREADS = 1024, WAVES = THREADS / 64, MOST_TILES = 256, ONE_TILE = 8;  // rounds of a sort in one launch

struct Sort {
    const int32_t* expert;
    int32_t *offsets, *place, *counts;  // counts [tiles][experts]
    int n, experts, tiles, rounds;
};
// The expert of assignment i, or -1
__device__ __forceinline__ int expert_of(const Sort& s, int64_t i)
{
    if (i >= s.n) return -1;
    const int e = s.expert[i];
    return (unsigned)e < (unsigned)s.experts ? e : -1;
}

__global__ __launch_bounds__(THREADS) void sort_count_kernel(Sort s)
{
    __shared__ int count[MOST_EXPERTS];
    for (int e = threadIdx.x; e < s.experts; e += THREADS) count[e] = 0;
    __syncthreads();
    for (int r = 0; r < s.rounds; ++r) {
        const int e = expert_of(s, ((int64_t)blockIdx.x * s.rounds + r) * THREADS + threadIdx.x);
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s.experts; e += THREADS) s.counts[(int64_t)blockIdx.x * s.experts + e] = count[e];
}

__global__ __launch_bounds__(THREADS) void sort_place_kernel(Sort s)
{
    extern __shared__ int table[];  // [WAVES][experts]: a wave's count of each expert, then the next place for it
    __shared__ int all[MOST_EXPERTS], before[MOST_EXPERTS], sums[WAVES];
    const int lane = threadIdx.x & 63, w = threadIdx.x / 64, E = s.experts;
    int* mine = table + w * E;
    for (int i = threadIdx.x; i < WAVES * E; i += THREADS) table[i] = 0;
    all[threadIdx.x] = before[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * s.rounds * THREADS + (int64_t)w * s.rounds * 64 + lane;
    for (int r = 0; r < s.rounds; ++r) {
        const int e = expert_of(s, first + 64 * r);
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    if (s.tiles > 1) {
        int across = 1;  // threads along the experts: a power of two, the others along the tiles
        while (across < E) across *= 2;
        const int e = threadIdx.x & (across - 1), parts = THREADS / across;
        int sum = 0, sum_before = 0;
        if (e < E)
#pragma unroll 8
            for (int g = threadIdx.x / across; g < s.tiles; g += parts) {
                const int c = s.counts[(int64_t)g * E + e];
                sum += c;
                sum_before += g < (int)blockIdx.x ? c : 0;
            }
        if (sum) atomicAdd(&all[e], sum);
        if (sum_before) atomicAdd(&before[e], sum_before);
    }
    __syncthreads();
    // thread e: expert e
    const int e = threadIdx.x;
    int total = 0;
    if (s.tiles > 1) {
        total = all[e];
    } else if (e < E) {
        for (int v = 0; v < WAVES; ++v) total += table[v * E + e];
    }
    int upto = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d, 64);
        if (lane >= d) upto += v;
    }
    if (lane == 63) sums[w] = upto;
    __syncthreads();
    for (int v = 0; v < w; ++v) upto += sums[v];
    if (e < E) {
        int next = upto - total;
        if (blockIdx.x == 0) {
            s.offsets[e] = next;
            if (e == E - 1) s.offsets[E] = upto;
        }
        next += before[e];
        for (int v = 0; v < WAVES; ++v) {
            const int c = table[v * E + e];
            table[v * E + e] = next;
            next += c;
        }
    }
    __syncthreads();
    for (int r = 0; r < s.rounds; ++r) {
        const int64_t i = first + 64 * r;
        const int own = expert_of(s, i);
        uint64_t same = __ballot(own >= 0);  // the lanes with this lane's expert
        for (int b = 1; b < E; b *= 2) {
            const uint64_t set = __ballot((own & b) != 0);
            same &= (own & b) ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        if (i < s.n) s.place[i] = own < 0 ? -1 : mine[own] + rank;
        __builtin_amdgcn_wave_barrier();  // everyone has read its place
        if (own >= 0 && rank == 0) mine[own] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- rows -----------------------------------------------------------------------------------
// A wave takes CHUNK accesses of 16 bytes a lane of one row at a time: 1024 elements (bf16, us, 512 | 1024 | 2048 | 4096: sums over two places of 32768 tokens of
// 4096 141 | 128 | 138 | 151, the gradient of 60000 tokens of 1024 in four places 173 | 174 | 234 | 425; fp32, gradient of 20000 of 4096 in two,
// 316 with 256, 307 with 512, 297 with 1024).  The last access of a row may be cut off (WHOLE: none is).
constexpr int SMALL = 256;
template <class T> constexpr int chunk_of = sizeof(T);
template <bool WHOLE, int V, class T> __device__ __forceinline__ Vec<T, V> take(const T* p, int c, int hidden, bool once)
{
    if (WHOLE || c + V <= hidden) return once ? load_once<V>(p + c) : load<V>(p + c);
    Vec<T, V> v;
#pragma unroll
    for (int e = 0; e < V; ++e) v.e[e] = c + e < hidden ? p[c + e] : T(0);
    return v;
}
template <bool WHOLE, int V, class T> __device__ __forceinline__ void give(T* p, int c, int hidden, const Vec<T, V>& v)
{
    if (WHOLE || c + V <= hidden) {
        store_once(p + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < hidden) p[c + e] = v.e[e];
    }
}
struct Rows {
    const int32_t* place;
    const float* weight;  // or NULL
    int64_t rows, places;
    int top, hidden;
};
// Where assignment a is, or -1
__device__ __forceinline__ int64_t place_of(const Rows& s, int64_t a)
{
    const int p = s.place[a];
    return (unsigned)p < (uint64_t)s.places ? p : -1;
}
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }

// xs[place(t, j)] = x[t].  (Read through the caches, where the step before may have left it: 32768 tokens of 4096 to two places, sort included, 122 us again and
// again and 148 with rows that nothing has touched; past them 148 in both.)
template <class T, bool WHOLE> __global__ __launch_bounds__(SMALL) void gather_kernel(const T* X, T* Xs, Rows s, int chunks)
{
    constexpr int V = 16 / sizeof(T), CHUNK = chunk_of<T>;
    const int lane = threadIdx.x & 63;
    for (int64_t unit = (int64_t)blockIdx.x * (SMALL / 64) + wave_id(); unit < s.rows * chunks; unit += (int64_t)gridDim.x * (SMALL / 64)) {
        const int64_t t = unit / chunks;
        const int c0 = ((int)(unit - t * chunks) * CHUNK * 64 + lane) * V;
        Vec<T, V> x[CHUNK];
#pragma unroll
        for (int k = 0; k < CHUNK; ++k)
            if (c0 + k * 64 * V < s.hidden) x[k] = take<WHOLE, V>(X + t * s.hidden, c0 + k * 64 * V, s.hidden, false);
        for (int j = 0; j < s.top; ++j) {
            const int64_t p = place_of(s, t * s.top + j);
            if (p < 0) continue;
#pragma unroll
            for (int k = 0; k < CHUNK; ++k)
                if (c0 + k * 64 * V < s.hidden) give<WHOLE, V>(Xs + p * s.hidden, c0 + k * 64 * V, s.hidden, x[k]);
        }
    }
}

// y[t] = sum_j (w(t, j)) ys[place(t, j)] (+ r[t]).  32768 tokens of 4096 in bf16 from two places each 133 us, 6.1 TB/s; 10007 of 2560 from eight 94, 4.9.
template <class T, bool WEIGHTED, bool WHOLE> __global__ __launch_bounds__(SMALL) void combine_kernel(const T* Ys, const T* R, T* Y, Rows s, int chunks)
{
    constexpr int V = 16 / sizeof(T), CHUNK = chunk_of<T>;
    const int lane = threadIdx.x & 63;
    for (int64_t unit = (int64_t)blockIdx.x * (SMALL / 64) + wave_id(); unit < s.rows * chunks; unit += (int64_t)gridDim.x * (SMALL / 64)) {
        const int64_t t = unit / chunks;
        const int c0 = ((int)(unit - t * chunks) * CHUNK * 64 + lane) * V;
        float sum[CHUNK][V] = {};
        for (int j = 0; j < s.top; ++j) {
            const int64_t p = place_of(s, t * s.top + j);
            if (p < 0) continue;
            const float w = WEIGHTED ? s.weight[t * s.top + j] : 1.f;
            Vec<T, V> y[CHUNK];
#pragma unroll
            for (int k = 0; k < CHUNK; ++k)
                if (c0 + k * 64 * V < s.hidden) y[k] = take<WHOLE, V>(Ys + p * s.hidden, c0 + k * 64 * V, s.hidden, true);
#pragma unroll
            for (int k = 0; k < CHUNK; ++k)
                if (c0 + k * 64 * V < s.hidden)
#pragma unroll
                    for (int e = 0; e < V; ++e) sum[k][e] = WEIGHTED ? fmaf(w, to_float(y[k].e[e]), sum[k][e]) : sum[k][e] + to_float(y[k].e[e]);
        }
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const int c = c0 + k * 64 * V;
            if (c >= s.hidden) continue;
            if (R) {
                const Vec<T, V> r = take<WHOLE, V>(R + t * s.hidden, c, s.hidden, true);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[k][e] += to_float(r.e[e]);
            }
            give<WHOLE, V>(Y + t * s.hidden, c, s.hidden, rounded<V>(sum[k], T()));
        }
    }
}

// dys[place(t, j)] = w(t, j) dy[t],  dw(t, j) = dy[t] . ys[place(t, j)].  (10007 tokens of 2560 in bf16, eight places: 157-165 us, 5.3 TB/s; eight waves a
// workgroup 160; ys through the caches 174.)  A wave takes an assignment at a time, a workgroup those of `tokens` neighbouring
// tokens, so that a row of dy comes from the memory once.  (The grid is bounded as the others' are: of a launch of 2^32 threads and more, those beyond
// do not run, without an error.)
template <class T, bool WHOLE>
__global__ __launch_bounds__(SMALL) void combine_bwd_kernel(const T* Ys, const T* dY, T* dYs, float* dweight, Rows s, int tokens)
{
    constexpr int V = 16 / sizeof(T), CHUNK = chunk_of<T>;
    const int lane = threadIdx.x & 63;
    for (int64_t token = (int64_t)blockIdx.x * tokens; token < s.rows; token += (int64_t)gridDim.x * tokens) {
        const int64_t first = token * s.top, end = first + (int64_t)tokens * s.top, last = end < s.rows * s.top ? end : s.rows * s.top;
        for (int64_t a = first + wave_id(); a < last; a += SMALL / 64) {
            const int64_t t = a / s.top, p = place_of(s, a);
            if (p < 0) {
                if (dweight && lane == 0) dweight[a] = 0.f;
                continue;
            }
            const float w = dYs ? s.weight[a] : 0.f;
            float dot = 0.f;
            for (int c0 = lane * V; c0 < s.hidden; c0 += CHUNK * 64 * V) {
                Vec<T, V> dy[CHUNK], y[CHUNK];
#pragma unroll
                for (int k = 0; k < CHUNK; ++k) {
                    const int c = c0 + k * 64 * V;
                    if (c >= s.hidden) continue;
                    dy[k] = take<WHOLE, V>(dY + t * s.hidden, c, s.hidden, false);
                    if (dweight) y[k] = take<WHOLE, V>(Ys + p * s.hidden, c, s.hidden, true);
                }
#pragma unroll
                for (int k = 0; k < CHUNK; ++k) {
                    const int c = c0 + k * 64 * V;
                    if (c >= s.hidden) continue;
                    if (dweight)
#pragma unroll
                        for (int e = 0; e < V; ++e) dot = fmaf(to_float(dy[k].e[e]), to_float(y[k].e[e]), dot);
                    if (dYs) {
                        float d[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) d[e] = w * to_float(dy[k].e[e]);
                        give<WHOLE, V>(dYs + p * s.hidden, c, s.hidden, rounded<V>(d, T()));
                    }
                }
            }
            if (dweight) {
                dot = lanes_sum<64>(dot);
                if (lane == 0) dweight[a] = dot;
            }
        }
    }
}

// ---- host side --------------------------------------------------------------------------------
Sort sort_of(int64_t n, int experts)
{
    Sort s = {};
    s.n = (int)n, s.experts = experts;
    if (n <= ONE_TILE * THREADS) {
        s.rounds = (int)((n + THREADS - 1) / THREADS), s.tiles = 1;
    } else {
        s.rounds = (int)((n + (int64_t)MOST_TILES * THREADS - 1) / ((int64_t)MOST_TILES * THREADS));
        s.tiles = (int)((n + (int64_t)s.rounds * THREADS - 1) / ((int64_t)s.rounds * THREADS));
    }
    return s;
}
int check_sort(int64_t n, int experts)
{
    if (n <= 0 || experts <= 0) return fail(TW_INVALID, "rows, top and experts must be positive");
    if (n > INT32_MAX || experts > MOST_EXPERTS) return fail(TW_UNSUPPORTED, "experts=%d beyond %d, or rows top beyond the launch limits", experts, MOST_EXPERTS);
    return TW_OK;
}
int check_rows(int64_t rows, int top, int hidden, int dtype)
{
    if (rows <= 0 || top <= 0 || hidden <= 0) return fail(TW_INVALID, "rows, top and hidden must be positive");
    if (dtype != FPDT_TW_F32 && dtype != FPDT_TW_BF16) return fail(TW_INVALID, "unknown dtype %d", dtype);
    if (rows > INT32_MAX || rows * top > INT32_MAX || hidden > 1 << 28) return fail(TW_UNSUPPORTED, "sizes beyond the launch limits");
    return TW_OK;
}
// Nothing that is written meets anything else, but where it is the very tensor number `same` of `in` (and that alone).
struct Arg {
    const void* p;
    size_t bytes;
};
bool meets(const Arg& out, const Arg* in, int n, int same = -1)
{
    for (int i = 0; i < n; ++i)
        if (out.p && in[i].p && !(i == same && in[i].p == out.p) && ranges_meet(out.p, out.bytes, in[i].p, in[i].bytes)) return true;
    return false;
}
// f(element type, WHOLE)
template <class F> void by_type(int dtype, int hidden, F f)
{
    if (dtype == FPDT_TW_F32) {
        if (hidden % 4 == 0) f(float(), std::true_type());
        else f(float(), std::false_type());
    } else {
        if (hidden % 8 == 0) f(uint16_t(), std::true_type());
        else f(uint16_t(), std::false_type());
    }
}
int chunks_of(int hidden) { return (hidden + 1023) / 1024; }  // (1024 elements in either type)
unsigned unit_grid(int64_t units)
{
    const int64_t n = (units + SMALL / 64 - 1) / (SMALL / 64);
    return (unsigned)(n < 1 << 20 ? n : 1 << 20);
}

// sum_j (weight) In[place] + R: combine's forward, gather's backward
int gathered_sum(const void* In, const float* weight, const int32_t* place, const void* R, void* Out, int64_t rows, int top, int hidden, int dtype, bool weighted,
                 hipStream_t st)
{
    clear_error();
    if (!In || !place || !Out || (weighted && !weight)) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_rows(rows, top, hidden, dtype);
    if (rc != TW_OK) return rc;
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, one = (size_t)rows * hidden * size, index = (size_t)rows * top * 4;
    if (misaligned(In, size) || misaligned(R, size) || misaligned(Out, size) || misaligned(place, 4) || misaligned(weight, 4))
        return fail(TW_INVALID, "a tensor is not aligned to its elements");
    const Arg in[] = {{In, one * top}, {weight, index}, {place, index}, {R, one}};
    if (meets({Out, one}, in, 4, 3)) return fail(TW_INVALID, "the output overlaps another tensor");
    const Rows s = {place, weight, rows, rows * top, top, hidden};
    const int chunks = chunks_of(hidden);
    by_type(dtype, hidden, [&](auto type, auto whole) {
        typedef decltype(type) T;
        constexpr bool WHOLE = decltype(whole)::value;
        const unsigned grid = unit_grid(rows * chunks);
        if (weighted) combine_kernel<T, true, WHOLE><<<grid, SMALL, 0, st>>>(static_cast<const T*>(In), static_cast<const T*>(R), static_cast<T*>(Out), s, chunks);
        else combine_kernel<T, false, WHOLE><<<grid, SMALL, 0, st>>>(static_cast<const T*>(In), static_cast<const T*>(R), static_cast<T*>(Out), s, chunks);
    });
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // namespace

extern "C" {

size_t fpdt_tw_experts_sort_workspace_bytes(int64_t assignments, int experts)
{
    if (assignments <= 0 || experts <= 0 || assignments > INT32_MAX || experts > MOST_EXPERTS) return 0;
    const Sort s = sort_of(assignments, experts);
    return s.tiles > 1 ? (size_t)s.tiles * experts * 4 : 256;
}

int fpdt_tw_experts_sort(const int32_t* expert, int32_t* offsets, int32_t* place, int64_t rows, int top, int experts, void* workspace, size_t workspace_bytes,
                         void* stream)
{
    clear_error();
    if (!expert || !offsets || !place) return fail(TW_INVALID, "NULL tensor pointer");
    if (rows <= 0 || top <= 0) return fail(TW_INVALID, "rows, top and experts must be positive");
    if (rows > INT32_MAX) return fail(TW_UNSUPPORTED, "rows beyond the launch limits");
    int rc = check_sort(rows * top, experts);
    if (rc != TW_OK) return rc;
    if (misaligned(expert, 4) || misaligned(offsets, 4) || misaligned(place, 4)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    const size_t need = fpdt_tw_experts_sort_workspace_bytes(rows * top, experts), index = (size_t)rows * top * 4, ends = (size_t)(experts + 1) * 4;
    if (!workspace || workspace_bytes < need || misaligned(workspace, 256))
        return fail(TW_WORKSPACE, "workspace NULL, misaligned or too small (%zu < %zu bytes)", workspace_bytes, need);
    const Arg every[] = {{expert, index}, {offsets, ends}, {place, index}, {workspace, need}};
    for (int i = 1; i < 4; ++i)
        if (meets(every[i], every, i)) return fail(TW_INVALID, "an output or the workspace overlaps another tensor");
    Sort s = sort_of(rows * top, experts);
    s.expert = expert, s.offsets = offsets, s.place = place, s.counts = static_cast<int32_t*>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (s.tiles > 1) sort_count_kernel<<<s.tiles, THREADS, 0, st>>>(s);
    sort_place_kernel<<<s.tiles, THREADS, (size_t)WAVES * experts * 4, st>>>(s);
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

int fpdt_tw_experts_gather_fwd(const void* X, const int32_t* place, void* Xs, int64_t rows, int top, int hidden, int dtype, void* stream)
{
    clear_error();
    if (!X || !place || !Xs) return fail(TW_INVALID, "NULL tensor pointer");
    int rc = check_rows(rows, top, hidden, dtype);
    if (rc != TW_OK) return rc;
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, one = (size_t)rows * hidden * size;
    if (misaligned(X, size) || misaligned(Xs, size) || misaligned(place, 4)) return fail(TW_INVALID, "a tensor is not aligned to its elements");
    const Arg in[] = {{X, one}, {place, (size_t)rows * top * 4}};
    if (meets({Xs, one * top}, in, 2)) return fail(TW_INVALID, "Xs overlaps another tensor");
    const Rows s = {place, nullptr, rows, rows * top, top, hidden};
    const int chunks = chunks_of(hidden);
    hipStream_t st = static_cast<hipStream_t>(stream);
    by_type(dtype, hidden, [&](auto type, auto whole) {
        typedef decltype(type) T;
        gather_kernel<T, decltype(whole)::value><<<unit_grid(rows * chunks), SMALL, 0, st>>>(static_cast<const T*>(X), static_cast<T*>(Xs), s, chunks);
    });
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

int fpdt_tw_experts_gather_bwd(const void* dXs, const int32_t* place, const void* R, void* dX, int64_t rows, int top, int hidden, int dtype, void* stream)
{
    return gathered_sum(dXs, nullptr, place, R, dX, rows, top, hidden, dtype, false, static_cast<hipStream_t>(stream));
}

int fpdt_tw_experts_combine_fwd(const void* Ys, const float* weight, const int32_t* place, const void* R, void* Y, int64_t rows, int top, int hidden, int dtype,
                                void* stream)
{
    return gathered_sum(Ys, weight, place, R, Y, rows, top, hidden, dtype, true, static_cast<hipStream_t>(stream));
}

int fpdt_tw_experts_combine_bwd(const void* Ys, const float* weight, const int32_t* place, const void* dY, void* dYs, float* dweight, int64_t rows, int top,
                                int hidden, int dtype, void* stream)
{
    clear_error();
    if (!place || !dY) return fail(TW_INVALID, "NULL tensor pointer");
    if (!dYs && !dweight) return fail(TW_INVALID, "nothing to compute: dYs and dweight are NULL");
    if ((dweight && !Ys) || (dYs && !weight)) return fail(TW_INVALID, "dweight needs Ys, and dYs needs weight");
    int rc = check_rows(rows, top, hidden, dtype);
    if (rc != TW_OK) return rc;
    const size_t size = dtype == FPDT_TW_F32 ? 4 : 2, one = (size_t)rows * hidden * size, index = (size_t)rows * top * 4;
    if (misaligned(Ys, size) || misaligned(dY, size) || misaligned(dYs, size) || misaligned(place, 4) || misaligned(weight, 4) || misaligned(dweight, 4))
        return fail(TW_INVALID, "a tensor is not aligned to its elements");
    const Arg in[] = {{Ys, one * top}, {weight, index}, {place, index}, {dY, one}, {dYs, one * top}};
    if (meets({dYs, one * top}, in, 4, 0) || meets({dweight, index}, in, 5)) return fail(TW_INVALID, "dYs or dweight overlaps another tensor");
    const Rows s = {place, weight, rows, rows * top, top, hidden};
    const int tokens = top < SMALL / 64 ? SMALL / 64 / top : 1;
    const int64_t groups = (rows + tokens - 1) / tokens;
    const unsigned grid = (unsigned)(groups < 1 << 20 ? groups : 1 << 20);
    hipStream_t st = static_cast<hipStream_t>(stream);
    by_type(dtype, hidden, [&](auto type, auto whole) {
        typedef decltype(type) T;
        combine_bwd_kernel<T, decltype(whole)::value><<<grid, SMALL, 0, st>>>(static_cast<const T*>(Ys), static_cast<const T*>(dY), static_cast<T*>(dYs), dweight, s,
                                                                              tokens);
    });
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // extern "C"
