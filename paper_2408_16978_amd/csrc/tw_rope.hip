// Rotary positions and the split of the QKV product (include/fpdt_tokenwise.h: fpdt_tw_rope_*).
//
// Channels (a, b) of a pair i at position p become A (a cos t - b sin t, b cos t + a sin t), t = p f_i; the gradient is
// the same with -t.  Every element is read once and written once: bound by the memory.
//
// The angle is formed in 64 bits (at 2M tokens a 32-bit product is off by 0.1 rad), turned into turns and reduced to an
// eighth of a turn there; sine and cosine of what is left are polynomials in 32 bits.  That is about 50 instructions a
// pair, so a thread keeps its pairs' sines and cosines for all heads that it turns of its token: no table is read from memory.
#include <cmath>

#include "../../include/fpdt_tokenwise.h"
#include "tw_common.h"

namespace {

using namespace fpdt_tw;

// What a wave of rope_any_kernel handles at a time of a tensor: `heads` heads of each of `tokens` tokens; per_token units to get
// through a token's heads (then tokens is 1).  by_*: 2^16 or 2^32 over a divisor, rounded up, in place of a quotient of numbers below 2^9,
// or of units.
struct Unit {
    int tokens, heads, per_token;
    int by_heads, by_tokens;
    unsigned by_units;
};

struct RopeArgs {
    const void* in[3];   // Q, K, V
    void* out[3];
    int64_t in_row[3], out_row[3];  // elements from a token to the next
    int heads[3];
    const int64_t* positions;
    int64_t position0, rows;
    const double* freqs;
    float amplitude, sign;  // sign: -1 in the backward
    int D, rot;
    int slots, head_lanes, tokens;  // slots of a head, heads and tokens of a workgroup at a time
    int split;          // heads of a workgroup (of all three tensors together)
    int by_access, by_pairs;
    Unit unit[3];
};

// sin and cos of 2 pi x, times `amplitude`.  x is reduced to within 1/8 of a multiple of 1/4 and made an angle in 64 bits, which is rounded once; the
// remainders of the Taylor series up to z^9 and z^10 at z = pi / 4 are below 2e-9 and 2e-10.  Right to 8e-8: half a step of the angle (3e-8 times at most 0.9), half
// a step of the result, 2e-8 of the sums before it (1e-7 with the reduced x rounded, and then its product with 2 pi).
__device__ __forceinline__ void sincos_turns(double x, float amplitude, float& s, float& c)
{
    x -= rint(x);
    const double k = rint(4. * x);
    const float z = (float)(6.2831853071795864769 * fma(-0.25, k, x)), z2 = z * z;
    const float ps = fmaf(z * z2, fmaf(z2, fmaf(z2, fmaf(z2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), z);
    const float pc = fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const int q = (int)k & 3;  // quarter turns
    const float ss = q & 1 ? pc : ps, cc = q & 1 ? ps : pc;
    s = amplitude * (q & 2 ? -ss : ss);
    c = amplitude * ((q + 1) & 2 ? -cc : cc);
}

// A slot of a head: V pairs in two accesses of V elements (halves; both layouts at V = 1), V / 2 pairs in one access
// (interleaved, V > 1), and behind the rotated channels V elements that are copied.
// LINES: what neighbouring lanes access are whole cache lines, which then go past the caches (us for those through them, bf16: 256K tokens, 1 / 1
// heads of 128 in halves 69 for 77, 4 / 4 heads of 80 interleaved 161 for 170; where they are not lines, 4 / 4 of 80 in halves, 245 for 195).
template <class T, int V, bool INTERLEAVED, bool LINES> __global__ __launch_bounds__(256) void rope_kernel(RopeArgs a)
{
    constexpr bool ONE = INTERLEAVED && V > 1;
    constexpr int PAIRS = ONE ? V / 2 : V, ACC = ONE ? 1 : 2, U = 4;
    const int turning = ONE ? a.rot / V : a.rot / 2 / V;
    const int hl = threadIdx.x / a.slots % a.head_lanes, lane = threadIdx.x / (a.slots * a.head_lanes);  // head of its kind, token of the workgroup
    const int h0 = blockIdx.y * a.split;
    auto get = [](const T* p) { return LINES ? load_once<V>(p) : load<V>(p); };
    auto put = [](T* p, const Vec<T, V>& v) {
        if (LINES) store_once(p, v);
        else store(p, v);
    };
    for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.rows; t0 += (int64_t)gridDim.x * a.tokens) {
        const int64_t row = t0 + lane;
        if (lane >= a.tokens || row >= a.rows) continue;
        const int64_t pos = a.positions ? a.positions[row] : a.position0 + row;
        for (int j = threadIdx.x % a.slots; j < a.slots; j += 256) {
            const bool turns = j < turning;
            float sn[PAIRS], cs[PAIRS];
            int at[2];
            if (turns) {
                at[0] = (INTERLEAVED && V == 1 ? 2 : 1) * j * V;
                at[1] = INTERLEAVED ? at[0] + 1 : at[0] + a.rot / 2;
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const double angle = (double)pos * a.freqs[j * PAIRS + i];
                    sincos_turns(angle * 0.15915494309189533577, a.amplitude, sn[i], cs[i]);
                    sn[i] *= a.sign;
                }
            } else {
                at[0] = at[1] = a.rot + (j - turning) * V;
            }
            int before = 0;
#pragma unroll
            for (int t = 0; t < 3; ++t) {
                // heads [from, to) of this tensor belong to the workgroup
                const int from = max(h0 - before, 0), to = min(h0 + a.split - before, a.heads[t]);
                before += a.heads[t];
                const bool turn = turns && t < 2;
                const T* in = static_cast<const T*>(a.in[t]) + row * a.in_row[t];
                T* out = static_cast<T*>(a.out[t]) + row * a.out_row[t];
                for (int h = from + hl; h < to; h += U * a.head_lanes) {
                    Vec<T, V> x[U][ACC];
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int c = 0; c < ACC; ++c)
                            if (h + u * a.head_lanes < to && (c == 0 || turns)) x[u][c] = get(in + (int64_t)(h + u * a.head_lanes) * a.D + at[c]);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (h + u * a.head_lanes >= to) break;
                        if (turn) {
                            float y[ACC * V];
#pragma unroll
                            for (int i = 0; i < PAIRS; ++i) {
                                const int ia = ONE ? 2 * i : i, ib = ONE ? 2 * i + 1 : V + i;
                                const float p = to_float(x[u][0].e[ia]), q = to_float(x[u][ib / V].e[ib % V]);
                                y[ia] = fmaf(p, cs[i], -q * sn[i]);
                                y[ib] = fmaf(q, cs[i], p * sn[i]);
                            }
#pragma unroll
                            for (int c = 0; c < ACC; ++c) x[u][c] = rounded<V>(y + c * V, T());
                        }
#pragma unroll
                        for (int c = 0; c < ACC; ++c)
                            if (c == 0 || turns) put(out + (int64_t)(h + u * a.head_lanes) * a.D + at[c], x[u][c]);
                    }
                }
            }
        }
    }
}

// Halves in accesses of 16 bytes: a lane has one access of a head, its pairs' other channels are in the lane `half / V` further.  What a
// wave accesses lies together then, whatever D is.  The two lanes share their pairs' sines and cosines: each forms half of them.  64K tokens, 32 / 8 heads
// of 128 257 us, 270 with a lane's halves in two accesses; 256K tokens, 8 / 2 of 64 131 for 147, 12 / 12 of 64 392 for 453, 4 / 4 of 80 177 for 194.
// Past the caches in whole lines as above: 32 / 8 of 128 257 for 292.
template <class T, bool LINES> __global__ __launch_bounds__(256) void rope_halves_kernel(RopeArgs a)
{
    constexpr int V = 16 / sizeof(T), H = V / 2, U = 4;
    typedef Vec<T, V> Access;
    const int lane = threadIdx.x & 63, sub = lane * a.by_access >> 16, acc = lane - sub * a.slots;  // head of the wave's, access of the head
    const int per_wave = 64 / a.slots, group = threadIdx.x / 64 * per_wave + sub, token = group / a.head_lanes, hl = group % a.head_lanes;
    const int far = a.rot / 2 / V, h0 = blockIdx.y * a.split;
    const bool turns = acc < 2 * far, low = acc < far;
    const int other = 4 * (lane + (low ? far : turns ? -far : 0));
    auto swap = [&](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(other, __builtin_bit_cast(int, x))); };
    auto get = [](const T* p) { return LINES ? load_once<V>(p) : load<V>(p); };
    auto put = [](T* p, const Vec<T, V>& v) {
        if (LINES) store_once(p, v);
        else store(p, v);
    };
    for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.rows; t0 += (int64_t)gridDim.x * a.tokens) {
        const int64_t row = t0 + token;
        if (sub >= per_wave || token >= a.tokens || row >= a.rows) continue;  // (a head's lanes all the same)
        const int64_t pos = a.positions ? a.positions[row] : a.position0 + row;
        float sn[V], cs[V];
        if (turns) {
            const int p0 = (low ? acc : acc - far) * V + (low ? 0 : H);
            float s[H], c[H];
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const double angle = (double)pos * a.freqs[p0 + i];
                sincos_turns(angle * 0.15915494309189533577, a.amplitude, s[i], c[i]);
                s[i] *= a.sign;
            }
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const float so = swap(s[i]), co = swap(c[i]);
                sn[i] = low ? s[i] : so, sn[H + i] = low ? so : s[i];
                cs[i] = low ? c[i] : co, cs[H + i] = low ? co : c[i];
            }
        }
        int before = 0;
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            // heads [from, to) of this tensor belong to the workgroup
            const int from = max(h0 - before, 0), to = min(h0 + a.split - before, a.heads[t]);
            before += a.heads[t];
            const T* in = static_cast<const T*>(a.in[t]) + row * a.in_row[t] + acc * V;
            T* out = static_cast<T*>(a.out[t]) + row * a.out_row[t] + acc * V;
            for (int h = from + hl; h < to; h += U * a.head_lanes) {
                Vec<T, V> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (h + u * a.head_lanes < to) x[u] = get(in + (int64_t)(h + u * a.head_lanes) * a.D);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (h + u * a.head_lanes >= to) break;
                    if (t < 2 && turns) {
                        uintx4 words = __builtin_bit_cast(uintx4, x[u]);
                        const unsigned flip = low ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0;  // a cos - b sin, b cos + a sin
#pragma unroll
                        for (int i = 0; i < 4; ++i) words[i] = (unsigned)__builtin_amdgcn_ds_bpermute(other, (int)words[i]) ^ flip;
                        const Vec<T, V> o = __builtin_bit_cast(Access, words);
                        float y[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) y[e] = fmaf(to_float(x[u].e[e]), cs[e], to_float(o.e[e]) * sn[e]);
                        x[u] = rounded<V>(y, T());
                    }
                    put(out + (int64_t)(h + u * a.head_lanes) * a.D, x[u]);
                }
            }
        }
    }
}

// Where 16 bytes do not fit the pairs (half of rot is odd, or twice an odd number): a workgroup turns `tokens` tokens.  A head is A = D / V accesses
// in neighbouring lanes, and a wave's 64 / A heads lie one behind the other in memory (those of one token, or of several
// where these have fewer).  Which token and which heads come next is the same for the wave; a lane's place among them never changes.
// Partners at a distance come through LDS; sines and cosines of the tile are formed once, in LDS, under the first loads.  65536 tokens, 8 / 2 heads of
// 128, rot = 30 in halves: 78 us, 182 with slots of one element; with slots of four (heads of 80, rot = 40) these are as fast, 122 us for 130.
constexpr int TABLE = 2048;  // pairs of a tile: 16 KB
// What lanes of a wave leave in LDS for each other.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <class T, bool INTERLEAVED> __global__ __launch_bounds__(256) void rope_any_kernel(RopeArgs a)
{
    constexpr int V = 16 / sizeof(T), U = 4;
    typedef Vec<T, V> Access;
    __shared__ float2 table[TABLE];  // cosine and sine
    __shared__ uintx4 tile[INTERLEAVED ? 1 : 256];
    const int A = a.D / V, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int sub = lane * a.by_access >> 16, acc = lane - sub * A;  // head of the wave's, access of the head
    const int half = a.rot / 2;

    // a lane's place in a unit of each tensor: token, head, and where it reads and writes
    int dtoken[3], dhead[3], lane_in[3], lane_out[3];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
        dtoken[t] = a.unit[t].tokens > 1 ? sub * a.unit[t].by_heads >> 16 : 0;
        dhead[t] = sub - dtoken[t] * a.heads[t];
        lane_in[t] = dtoken[t] * (int)a.in_row[t] + dhead[t] * a.D + acc * V;
        lane_out[t] = dtoken[t] * (int)a.out_row[t] + dhead[t] * a.D + acc * V;
        if (sub >= a.unit[t].tokens * a.unit[t].heads) dhead[t] = 1 << 20;  // no place: no head
    }
    auto pick = [](int t, auto x, auto y, auto z) { return t == 0 ? x : t == 1 ? y : z; };
    const T *in0 = static_cast<const T*>(a.in[0]), *in1 = static_cast<const T*>(a.in[1]), *in2 = static_cast<const T*>(a.in[2]);
    T *out0 = static_cast<T*>(a.out[0]), *out1 = static_cast<T*>(a.out[1]), *out2 = static_cast<T*>(a.out[2]);
    const int in_row0 = (int)a.in_row[0], in_row1 = (int)a.in_row[1], in_row2 = (int)a.in_row[2];
    const int out_row0 = (int)a.out_row[0], out_row1 = (int)a.out_row[1], out_row2 = (int)a.out_row[2];
    const Unit n0 = a.unit[0], n1 = a.unit[1], n2 = a.unit[2];
    for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.rows; t0 += (int64_t)gridDim.x * a.tokens) {
        const int tokens = (int)min((int64_t)a.tokens, a.rows - t0);
        // units of the tile, tensor by tensor
        const int end0 = ((tokens + n0.tokens - 1) * n0.by_tokens >> 16) * n0.per_token;
        const int end1 = end0 + ((tokens + n1.tokens - 1) * n1.by_tokens >> 16) * n1.per_token;
        const int n = end1 + ((tokens + n2.tokens - 1) * n2.by_tokens >> 16) * n2.per_token;
        Access x[U];
        bool here[U];
        int tensor[U], token[U], head[U];  // of the unit
        auto fetch = [&](int unit0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int unit = unit0 + u * 4 + wave, t = unit < end0 ? 0 : unit < end1 ? 1 : 2;
                const int k = unit - pick(t, 0, end0, end1), per = pick(t, n0.per_token, n1.per_token, n2.per_token);
                const int row = per == 1 ? k : (int)__umulhi(k, pick(t, n0.by_units, n1.by_units, n2.by_units));
                tensor[u] = t, token[u] = row * pick(t, n0.tokens, n1.tokens, n2.tokens), head[u] = (k - row * per) * pick(t, n0.heads, n1.heads, n2.heads);
                here[u] = unit < n && token[u] + pick(t, dtoken[0], dtoken[1], dtoken[2]) < tokens
                    && head[u] + pick(t, dhead[0], dhead[1], dhead[2]) < pick(t, a.heads[0], a.heads[1], a.heads[2]);
                const int64_t row_in = pick(t, in_row0, in_row1, in_row2);
                const T* in = pick(t, in0, in1, in2) + (t0 + token[u]) * row_in + head[u] * a.D;
                if (here[u]) x[u] = load_once<V>(in + (unsigned)pick(t, lane_in[0], lane_in[1], lane_in[2]));
            }
        };
        fetch(0);
        const int wide = 256 * a.by_pairs >> 16;  // tokens at once: a thread keeps its pair
        const int tk = threadIdx.x * a.by_pairs >> 16, p = threadIdx.x - tk * half;
        if (tk < wide) {
            const double f = a.freqs[p];
            for (int k = tk; k < tokens; k += wide) {
                const int64_t pos = a.positions ? a.positions[t0 + k] : a.position0 + t0 + k;
                float sn, cs;
                sincos_turns((double)pos * f * 0.15915494309189533577, a.amplitude, sn, cs);
                table[k * half + p] = make_float2(cs, a.sign * sn);
            }
        }
        __syncthreads();
        for (int unit0 = 0; unit0 < n; unit0 += 4 * U) {
            if (unit0) fetch(unit0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (unit0 + u * 4 + wave >= n) continue;
                const int t = tensor[u];
                if (t < 2) {
                    // (lanes without a place read what another token has, and write nothing)
                    const float2* tab = table + (here[u] ? token[u] + (t == 0 ? dtoken[0] : dtoken[1]) : 0) * half;
                    float y[V];
                    if constexpr (INTERLEAVED) {
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            const int c = acc * V + e;
                            y[e] = to_float(x[u].e[e]), y[e + 1] = to_float(x[u].e[e + 1]);
                            if (here[u] && c < a.rot) {
                                const float2 k = tab[c / 2];
                                const float p = y[e], q = y[e + 1];
                                y[e] = fmaf(p, k.x, -q * k.y), y[e + 1] = fmaf(q, k.x, p * k.y);
                            }
                        }
                    } else {
                        tile[threadIdx.x] = __builtin_bit_cast(uintx4, x[u]);
                        wave_sync();
                        const T* from = reinterpret_cast<const T*>(tile + threadIdx.x - acc);
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const int c = acc * V + e;
                            y[e] = to_float(x[u].e[e]);
                            if (here[u] && c < a.rot) {
                                const int i = c < half ? c : c - half;
                                const float2 k = tab[i];
                                const float other = to_float(from[c < half ? c + half : i]);
                                y[e] = fmaf(y[e], k.x, c < half ? -other * k.y : other * k.y);
                            }
                        }
                        wave_sync();
                    }
                    x[u] = rounded<V>(y, T());
                }
                const int64_t row_out = pick(t, out_row0, out_row1, out_row2);
                T* out = pick(t, out0, out1, out2) + (t0 + token[u]) * row_out + head[u] * a.D;
                if (here[u]) store_once(out + (unsigned)pick(t, lane_out[0], lane_out[1], lane_out[2]), x[u]);
            }
        }
        __syncthreads();  // the next tile's table
    }
}

constexpr int MOST_D = 8192, MOST_HEADS = 4096;

template <class T, int V> void launch_v(const RopeArgs& a, bool interleaved, bool lines, dim3 grid, hipStream_t st)
{
    if constexpr (V * sizeof(T) == 16) {
        if (lines && interleaved) rope_kernel<T, V, true, true><<<grid, 256, 0, st>>>(a);
        else if (lines) rope_kernel<T, V, false, true><<<grid, 256, 0, st>>>(a);
        if (lines) return;
    }
    if (interleaved) rope_kernel<T, V, true, false><<<grid, 256, 0, st>>>(a);
    else rope_kernel<T, V, false, false><<<grid, 256, 0, st>>>(a);
}

template <class T> void launch_any(RopeArgs& a, bool interleaved, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    const int per_wave = 64 / (a.D / V);
    auto by = [](int d) { return (65536 + d - 1) / d; };
    a.by_access = by(a.D / V), a.by_pairs = by(a.rot / 2);
    for (int t = 0; t < 3; ++t) {
        const int h = a.heads[t];
        Unit& n = a.unit[t];
        n.tokens = h && h < per_wave ? per_wave / h : 1;
        n.heads = h < per_wave ? h : per_wave;
        n.per_token = (h + per_wave - 1) / per_wave;
        n.by_heads = h ? by(h) : 0, n.by_tokens = by(n.tokens);
        n.by_units = n.per_token > 1 ? (unsigned)((0x100000000ull + n.per_token - 1) / n.per_token) : 0;
    }
    // Tokens of a tile: as many as 16 KB of sines and cosines are, 16 at most, and fewer until there are four workgroups for
    // each compute unit.
    a.tokens = TABLE / (a.rot / 2) < 16 ? TABLE / (a.rot / 2) : 16;
    while (a.tokens > 1 && a.rows / a.tokens < 1024) a.tokens = (a.tokens + 1) / 2;
    const int64_t tiles = (a.rows + a.tokens - 1) / a.tokens;
    const unsigned grid = (unsigned)(tiles < (1 << 20) ? tiles : 1 << 20);
    if (interleaved) rope_any_kernel<T, true><<<grid, 256, 0, st>>>(a);
    else rope_any_kernel<T, false><<<grid, 256, 0, st>>>(a);
}

// The widest access whose elements are all turned or all copied, in either half.
int access(int D, int rot, bool interleaved, int most)
{
    int v = most;
    while (v > 1 && ((interleaved ? rot : rot / 2) % v || (D - rot) % v)) v /= 2;
    return v;
}

// Do two tensors of rows of `wa` and `wb` bytes, `ra` and `rb` bytes apart, share a byte?  Rows of one distance may lie
// between each other; with two distances, ranges that meet count as shared.
bool rows_meet(const void* a, int64_t ra, int64_t wa, const void* b, int64_t rb, int64_t wb, int64_t rows)
{
    if (!ranges_meet(a, (size_t)((rows - 1) * ra + wa), b, (size_t)((rows - 1) * rb + wb))) return false;
    if (ra != rb) return rows > 1 || ranges_meet(a, (size_t)wa, b, (size_t)wb);
    if (rows == 1) return true;
    const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
    const int64_t m = ((d % ra) + ra) % ra;  // columns from a row of a to the next row of b
    return m < wa || ra - m < wb;
}

int rope(const void* const in[3], const int64_t in_row[3], void* const out[3], const int64_t out_row[3], const int64_t* positions, int64_t position0,
         const double* freqs, float amplitude, int64_t rows, int Hq, int Hkv, int D, int rot, int layout, int dtype, bool back, void* stream)
{
    clear_error();
    static const char* const names = "QKV";
    if (rows <= 0 || Hq <= 0 || Hkv < 0 || D <= 0) return fail(TW_INVALID, "rows, Hq and D must be positive, Hkv not negative");
    if (rot <= 0 || rot % 2 || rot > D) return fail(TW_INVALID, "rot=%d must be even and in [2, D]", rot);
    if (layout != FPDT_TW_ROPE_HALF && layout != FPDT_TW_ROPE_INTERLEAVED) return fail(TW_INVALID, "unknown layout %d", layout);
    if (dtype != FPDT_TW_F32 && dtype != FPDT_TW_BF16) return fail(TW_INVALID, "unknown dtype %d", dtype);
    if (!std::isfinite(amplitude)) return fail(TW_INVALID, "amplitude must be finite");
    if (!freqs || misaligned(freqs, 8) || misaligned(positions, 8)) return fail(TW_INVALID, "freqs NULL, or freqs or positions misaligned");
    if (D > MOST_D || Hq > MOST_HEADS || Hkv > MOST_HEADS || rows > INT32_MAX) return fail(TW_UNSUPPORTED, "sizes beyond the launch limits");
    const int size = dtype == FPDT_TW_F32 ? 4 : 2;
    RopeArgs a = {};
    for (int t = 0; t < 3; ++t) {
        const int heads = t == 0 ? Hq : Hkv;
        if ((in[t] == nullptr) != (out[t] == nullptr)) return fail(TW_INVALID, "%c is given on one side only", names[t]);
        if (!in[t]) {
            if (t == 0) return fail(TW_INVALID, "NULL tensor pointer");
            continue;
        }
        if (heads == 0) return fail(TW_INVALID, "%c is given, but Hkv is 0", names[t]);
        if (in_row[t] < (int64_t)heads * D || out_row[t] < (int64_t)heads * D) return fail(TW_INVALID, "rows of %c are closer than its heads are long", names[t]);
        if (in_row[t] > (1 << 28) || out_row[t] > (1 << 28)) return fail(TW_UNSUPPORTED, "rows of %c beyond the launch limits", names[t]);
        if (misaligned(in[t], size) || misaligned(out[t], size)) return fail(TW_INVALID, "%c is not aligned to its elements", names[t]);
        a.in[t] = in[t], a.out[t] = out[t], a.in_row[t] = in_row[t], a.out_row[t] = out_row[t], a.heads[t] = heads;
    }
    // what is written may be what is read at the same place, and nothing else
    for (int t = 0; t < 3; ++t)
        for (int u = 0; u < 3; ++u) {
            const int64_t wt = (int64_t)a.heads[t] * D * size, wu = (int64_t)a.heads[u] * D * size;
            if (!wt || !wu) continue;
            const bool same = t == u && a.out[t] == a.in[u] && a.out_row[t] == a.in_row[u];
            if (!same && rows_meet(a.out[t], a.out_row[t] * size, wt, a.in[u], a.in_row[u] * size, wu, rows))
                return fail(TW_INVALID, "%c's output overlaps %c's input", names[t], names[u]);
            if (t < u && rows_meet(a.out[t], a.out_row[t] * size, wt, a.out[u], a.out_row[u] * size, wu, rows))
                return fail(TW_INVALID, "the outputs of %c and %c overlap", names[t], names[u]);
        }
    a.positions = positions, a.position0 = position0, a.rows = rows, a.freqs = freqs, a.amplitude = amplitude, a.sign = back ? -1.f : 1.f;
    a.D = D, a.rot = rot;
    const bool inter = layout == FPDT_TW_ROPE_INTERLEAVED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int full = 16 / size, v = access(D, rot, inter, full), heads = a.heads[0] + a.heads[1] + a.heads[2];
    bool near = true;  // a tile's offsets fit 32 bits
    for (int t = 0; t < 3; ++t) near = near && in_row[t] <= (1 << 24) && out_row[t] <= (1 << 24);
    if (v <= full / 4 && D % full == 0 && D / full <= 64 && near) {
        if (size == 4) launch_any<float>(a, inter, st);
        else launch_any<uint16_t>(a, inter, st);
        HIP_TRY(hipGetLastError());
        return TW_OK;
    }
    a.slots = (inter && v > 1 ? rot / v : rot / 2 / v) + (D - rot) / v;
    // Halves in accesses of 16 bytes go through rope_halves_kernel, but for those of whole cache lines with so few heads that the exchange of the
    // sines shows (256K tokens, bf16, there | with two accesses a lane, us: 1 / 1 heads of 128 81 | 69, 2 / 2 131 | 131, back 136 | 131; 1 / 1 of 64 40 | 43,
    // 1 / 1 of 80 54 | 58).
    const bool halves = !inter && v == full && D / full <= 64 && (rot / 2 * size % 128 || heads > 6);
    if (halves) a.slots = D / full, a.by_access = (65536 + a.slots - 1) / a.slots;
    // Neighbouring lanes take neighbouring heads too, which keeps what a wave accesses together, up to where a third of the lanes has no head (64K
    // tokens, 32 / 8 heads of 128 interleaved, us with 1 | 2 | 4 | 8 of them: 290 | 281 | 272 | 260; 256K tokens, 4 / 4 of 80 191 | 177 | 170 | 243); in halves, where
    // sines and partners cost more, as long as a lane has six heads (64K, 32 / 8 of 128 294 | 284 | 276 | 257, 8 / 2 70 | 68 | 76; 256K, 8 / 2 of 64 140 | 131 | 148).
    a.head_lanes = 1;
    for (int n = 2; n <= 8 && n * a.slots <= 256; n *= 2) {
        int passes = 0;
        for (int h : a.heads) passes += (h + n - 1) / n;
        if (3 * n * passes <= 4 * heads && (!halves || passes >= 6)) a.head_lanes = n;
    }
    const int groups = halves ? 4 * (64 / a.slots) : a.slots >= 256 ? 1 : 256 / a.slots;  // heads of a workgroup at a time
    if (a.head_lanes > groups) a.head_lanes = groups >= 4 ? 4 : groups >= 2 ? 2 : 1;
    a.tokens = groups / a.head_lanes;
    // What the lanes of a token access: heads (interleaved), or a half and what is copied.
    bool lines = v == full && (inter || halves ? a.head_lanes : 1) * D * size % 128 == 0 && (inter || halves || rot / 2 * size % 128 == 0);
    for (int t = 0; t < 3; ++t)
        lines = lines && !misaligned(a.in[t], 128) && !misaligned(a.out[t], 128) && a.in_row[t] * size % 128 == 0 && a.out_row[t] * size % 128 == 0;
    const int64_t tiles = (rows + a.tokens - 1) / a.tokens;
    // All heads of a token in one workgroup, as long as that leaves every compute unit some of them.
    int parts = tiles >= 1024 ? 1 : (int)((1024 + tiles - 1) / tiles);
    if (parts > (heads + a.head_lanes - 1) / a.head_lanes) parts = (heads + a.head_lanes - 1) / a.head_lanes;
    a.split = (heads + parts - 1) / parts;
    const dim3 grid((unsigned)(tiles < (1 << 20) ? tiles : 1 << 20), (unsigned)((heads + a.split - 1) / a.split));
    if (halves) {
        if (size == 4 && lines) rope_halves_kernel<float, true><<<grid, 256, 0, st>>>(a);
        else if (size == 4) rope_halves_kernel<float, false><<<grid, 256, 0, st>>>(a);
        else if (lines) rope_halves_kernel<uint16_t, true><<<grid, 256, 0, st>>>(a);
        else rope_halves_kernel<uint16_t, false><<<grid, 256, 0, st>>>(a);
    } else if (size == 4) {
        if (v == 4) launch_v<float, 4>(a, inter, lines, grid, st);
        else if (v == 2) launch_v<float, 2>(a, inter, lines, grid, st);
        else launch_v<float, 1>(a, inter, lines, grid, st);
    } else {
        if (v == 8) launch_v<uint16_t, 8>(a, inter, lines, grid, st);
        else if (v == 4) launch_v<uint16_t, 4>(a, inter, lines, grid, st);
        else if (v == 2) launch_v<uint16_t, 2>(a, inter, lines, grid, st);
        else launch_v<uint16_t, 1>(a, inter, lines, grid, st);
    }
    HIP_TRY(hipGetLastError());
    return TW_OK;
}

}  // namespace

extern "C" {

int fpdt_tw_rope_freqs(int rot, double base, int scaling, double factor, double context, double low, double high, double* freqs)
{
    clear_error();
    if (!freqs) return fail(TW_INVALID, "NULL pointer");
    if (rot <= 0 || rot % 2 || rot > MOST_D) return fail(TW_INVALID, "rot=%d must be even and in [2, %d]", rot, MOST_D);
    if (!std::isfinite(base) || base <= 0) return fail(TW_INVALID, "base must be finite and positive");
    if (scaling < FPDT_TW_ROPE_PLAIN || scaling > FPDT_TW_ROPE_PARTS) return fail(TW_INVALID, "unknown scaling %d", scaling);
    if (scaling != FPDT_TW_ROPE_PLAIN && (!std::isfinite(factor) || factor <= 0)) return fail(TW_INVALID, "factor must be finite and positive");
    if (scaling == FPDT_TW_ROPE_PARTS && !(std::isfinite(context) && context > 0 && std::isfinite(low) && std::isfinite(high) && low < high))
        return fail(TW_INVALID, "by parts: context must be positive, and low < high");
    if (scaling == FPDT_TW_ROPE_RAISED && rot > 2) base *= std::pow(factor, rot / (rot - 2.));
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2. * i / rot);
        if (scaling == FPDT_TW_ROPE_LINEAR) f /= factor;
        if (scaling == FPDT_TW_ROPE_PARTS) {
            const double turns = context * f / 6.2831853071795864769;
            const double keep = std::fmin(1., std::fmax(0., (turns - low) / (high - low)));
            f = keep * f + (1 - keep) * f / factor;
        }
        freqs[i] = f;
    }
    return TW_OK;
}

int fpdt_tw_rope_fwd(const void* Q, int64_t q_row, const void* K, int64_t k_row, const void* V, int64_t v_row, void* Qo, int64_t qo_row, void* Ko,
                     int64_t ko_row, void* Vo, int64_t vo_row, const int64_t* positions, int64_t position0, const double* freqs, float amplitude,
                     int64_t rows, int Hq, int Hkv, int D, int rot, int layout, int dtype, void* stream)
{
    const void* const in[3] = {Q, K, V};
    void* const out[3] = {Qo, Ko, Vo};
    const int64_t in_row[3] = {q_row, k_row, v_row}, out_row[3] = {qo_row, ko_row, vo_row};
    return rope(in, in_row, out, out_row, positions, position0, freqs, amplitude, rows, Hq, Hkv, D, rot, layout, dtype, false, stream);
}

int fpdt_tw_rope_bwd(const void* dQo, int64_t qo_row, const void* dKo, int64_t ko_row, const void* dVo, int64_t vo_row, void* dQ, int64_t q_row,
                     void* dK, int64_t k_row, void* dV, int64_t v_row, const int64_t* positions, int64_t position0, const double* freqs,
                     float amplitude, int64_t rows, int Hq, int Hkv, int D, int rot, int layout, int dtype, void* stream)
{
    const void* const in[3] = {dQo, dKo, dVo};
    void* const out[3] = {dQ, dK, dV};
    const int64_t in_row[3] = {qo_row, ko_row, vo_row}, out_row[3] = {q_row, k_row, v_row};
    return rope(in, in_row, out, out_row, positions, position0, freqs, amplitude, rows, Hq, Hkv, D, rot, layout, dtype, true, stream);
}

}  // extern "C"
