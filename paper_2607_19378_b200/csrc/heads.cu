// Queries and keys as heads: the norm of each head and the rotation by its token's position on the grid, in one pass, and its gradient.
//
// q is [B][Hq D][T], k is [B][Hk D][T], T = L_1 .. L_N.  Per token and head, over its D channels:
//     x^ = x rho,  rho = 1 / sqrt(mean(x^2) + eps) | 1 / sqrt(sum(x^2) + eps) | 1,      n = x^ g,
//     y_i = n_i cos(t) - n_{i+D/2} sin(t),  y_{i+D/2} = n_i sin(t) + n_{i+D/2} cos(t)   for the pairs i that have an axis,
// t = p_a base^(-j / s_a) for the j-th of the s_a pairs of axis a, p_a the token's place on it.  Gradient: dn is dy turned back,
//     dg = sum dn x^,   dx = rho (e - x^ (e . x^) / D)  (rms; l2: without the division; none: e),   e = dn g.
//
// Each tensor is read and written once: bandwidth is the bound, instructions the next one.  Tokens are the contiguous axis, so a CTA takes a
// tile of 128 bytes of tokens and walks the heads and batch entries on it; a head's channels are spread over R groups of eight lanes (a
// lane holds 16 bytes of tokens of both channels of a pair), its sums go by shuffles and, beyond a warp, through shared memory.
// The tile's sines and cosines are formed once for all heads: angles as turns in 64 bits (in 32 a position of 100000 keeps two digits),
// reduced to half a turn and rounded.  On the grid's own positions few of them are: along the last axis a tile's first position
// turned on by those of 0, 1, 2 .. (kept for all tiles), along the others one for each row of the grid in the tile.  An error stays
// below 2e-7 at any position.  A grid of fewer than eight tokens (generation) goes to a warp per token and head.
#include <math.h>

#include "entry.cuh"
#include "octet.cuh"
#include "pair.cuh"

namespace hn {

enum { NORM_NONE = HYENAND_NORM_NONE, NORM_RMS = HYENAND_NORM_RMS, NORM_L2 = HYENAND_NORM_L2 };
constexpr int kMaxD = 256, kMaxAxes = 3;

struct HeadsArgs {
    const void *x[2], *dy[2];                // q and k
    void *out[2];
    const float *g[2];
    const int *positions;                    // [B][N][T], or the grid's
    float *part;                             // [blocks][2][D]: sums of the weights' gradients
    float *dg[2];
    int H[2], splits;
    int B, D, T, ndim, dims[kMaxAxes], axes[kMaxAxes], turned;
    int tiles, norm;
    float eps, per_mean;                     // 1/D, or 1: what a sum over channels counts
    double log2_base;
};

// cosine and sine of p base^(-j/s)
__device__ __forceinline__ float2 rotor(int p, double frequency)
{
    double turns = (double)p * frequency;
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    return make_float2(c, s);
}
// axis and turns per position of a pair
__device__ __forceinline__ double pair_frequency(const HeadsArgs &a, int i, int *axis)
{
    int n = 0;
    while (i >= a.axes[n]) i -= a.axes[n++];
    *axis = n;
    return exp2(-(double)i / a.axes[n] * a.log2_base) * 0.15915494309189533577;
}
__device__ __forceinline__ int place(const HeadsArgs &a, int b, int axis, int t)
{
    if (a.positions) {
        const int *p = a.positions + ((long long)b * a.ndim + axis) * a.T + t;
        HN_G(p, 4);
        return __ldg(p);
    }
    for (int n = a.ndim - 1; n > axis; --n) t /= a.dims[n];
    return axis ? t % a.dims[axis] : t;
}

template <typename T> struct Tile {
    static constexpr int V = 16 / sizeof(T), TOKENS = 8 * V;
};

// A token whose mean square is beyond fp32 though its channels are not is taken at this scale: then 256 squares of the largest number fit,
// and one that brought the mean there is still 2^-10.
constexpr float kShrink = 0x1p-70f, kLargest = 3.402823466e38f;

// The V tokens of a lane in one row, in pairs: side by side as one vector, or (rows that do not start on 16 bytes) every eighth token, so
// that the eight lanes of a row share a sector
template <typename T, bool VEC> struct Tokens {
    uint4 w;
    __device__ __forceinline__ void load(const T *row, int t0, int vc, int T_)
    {
        constexpr int V = Tile<T>::V;
        w = make_uint4(0, 0, 0, 0);
        if constexpr (VEC) {
            const int t = t0 + vc * V;
            if (t < T_) { HN_G(row + t, 16); w = __ldg((const uint4 *)(row + t)); }
        } else {
            unsigned x[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const T *p = row + t0 + i * 8 + vc;
                x[i] = 0;
                if (t0 + i * 8 + vc < T_) {
                    HN_G(p, sizeof(T));
                    if constexpr (sizeof(T) == 2) x[i] = __ldg((const unsigned short *)p);
                    else x[i] = __float_as_uint(__ldg((const float *)p));
                }
            }
            if constexpr (sizeof(T) == 2) w = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[V - 4] | x[V - 3] << 16, x[V - 2] | x[V - 1] << 16);
            else w = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
    __device__ __forceinline__ void get(f2 (&v)[Tile<T>::V / 2]) const
    {
        const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < Tile<T>::V / 2; ++i) v[i] = sizeof(T) == 2 ? widen2(u[i]) : make2(__uint_as_float(u[2 * i & 3]), __uint_as_float(u[(2 * i + 1) & 3]));
    }
};
// 1 / sqrt(v), the approximation set right by a step of Newton's method (two roundings; sqrt and division would be a third of a head's work)
__device__ __forceinline__ float inverse_root(float v)
{
    const float y = rsqrtf(v);
    return fmaf(0.5f * y, fmaf(-v * y, y, 1.f), y);
}
template <typename T, bool VEC> __device__ __forceinline__ void store_tokens(T *row, const f2 (&v)[Tile<T>::V / 2], int t0, int vc, int T_)
{
    constexpr int V = Tile<T>::V;
    if constexpr (VEC) {
        const int t = t0 + vc * V;
        uint4 w;
        if constexpr (sizeof(T) == 2) w = make_uint4(narrow2(v[0]), narrow2(v[1]), narrow2(v[V / 2 - 2]), narrow2(v[V / 2 - 1]));
        else w = make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
        if (t < T_) { HN_G(row + t, 16); *(uint4 *)(row + t) = w; }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (t0 + i * 8 + vc < T_) IO<T>::st(row, t0 + i * 8 + vc, i & 1 ? v[i / 2].y : v[i / 2].x);
    }
}

// where a lane's token e of a table's row lies: vectors of four, lane after lane
__device__ __forceinline__ int table_at(int lane, int element) { return (element / 4 * 8 + lane) * 4 + element % 4; }
template <typename T, bool VEC> __device__ __forceinline__ int token_at(int e) { return VEC ? table_at(e / Tile<T>::V, e % Tile<T>::V) : table_at(e % 8, e / 8); }

// The tile's table: cosines and sines [pair][token_at].  `steps`: the same of the positions 0 .. TOKENS - 1 for the pairs of the last axis,
// formed before; `rows`: room for rows_of_tile() rotors a pair.
__host__ __device__ __forceinline__ int rows_of_tile(int tokens, int last) { return last >= tokens ? 2 : (tokens - 1) / last + 2; }
template <typename T, bool VEC> __device__ __forceinline__ void fill_table(const HeadsArgs &a, int b, int t0, float *cs, float *sn, const float *step_c, const float *step_s, float2 *rows, const double *freq, const int *axis_of, int tid)
{
    constexpr int V = Tile<T>::V, TOKENS = Tile<T>::TOKENS;
    if (a.positions) {
        for (int i = tid; i < a.turned * TOKENS; i += 256) {
            const int pr = i / TOKENS, e = i % TOKENS;
            const float2 c = t0 + e < a.T ? rotor(place(a, b, axis_of[pr], t0 + e), freq[pr]) : make_float2(1.f, 0.f);
            cs[pr * TOKENS + token_at<T, VEC>(e)] = c.x;
            sn[pr * TOKENS + token_at<T, VEC>(e)] = c.y;
        }
        return;
    }
    // rotors of the rows of the grid that the tile touches (of the last axis: of its first position, the other rows start at 0)
    const int Ln = a.dims[a.ndim - 1], pitch = rows_of_tile(TOKENS, Ln), row0 = t0 / Ln, first = t0 - row0 * Ln, n = (t0 + TOKENS - 1) / Ln - row0 + 1;
    for (int i = tid; i < a.turned * n; i += 256) {
        const int pr = n == 1 ? i : i / n, k = n == 1 ? 0 : i % n, axis = axis_of[pr];
        float2 c = make_float2(1.f, 0.f);
        if (axis == a.ndim - 1) { if (k == 0) c = rotor(first, freq[pr]); }
        else {
            int r = row0 + k;
            for (int m = a.ndim - 2; m > axis; --m) r /= a.dims[m];
            c = rotor(axis ? r % a.dims[axis] : r, freq[pr]);
        }
        rows[pr * pitch + k] = c;
    }
    __syncthreads();
    if (n == 1) {                                                  // a lane's V tokens at a time
        for (int i = tid; i < a.turned * 8; i += 256) {
            const int pr = i >> 3;
            const float2 c = rows[pr * pitch];
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const int at = pr * TOKENS + table_at(i & 7, e);
                f2 x[2] = {pair(c.x), pair(c.x)}, y[2] = {pair(c.y), pair(c.y)};
                if (axis_of[pr] == a.ndim - 1) {
                    const float4 p = *(const float4 *)(step_c + at), q = *(const float4 *)(step_s + at);
                    const f2 u[2] = {make2(p.x, p.y), make2(p.z, p.w)}, w[2] = {make2(q.x, q.y), make2(q.z, q.w)};
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        x[m] = fma2(pair(c.x), u[m], mul2(pair(-c.y), w[m]));
                        y[m] = fma2(pair(c.x), w[m], mul2(pair(c.y), u[m]));
                    }
                }
                *(float4 *)(cs + at) = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
                *(float4 *)(sn + at) = make_float4(y[0].x, y[0].y, y[1].x, y[1].y);
            }
        }
        return;
    }
    for (int i = tid; i < a.turned * TOKENS; i += 256) {
        const int pr = i / TOKENS, e = i % TOKENS, at = pr * TOKENS + token_at<T, VEC>(e), k = (first + e) / Ln;
        float2 c = rows[pr * pitch + k];
        if (axis_of[pr] == a.ndim - 1) {
            const int from = pr * TOKENS + token_at<T, VEC>(k ? first + e - k * Ln : e);
            c = make_float2(c.x * step_c[from] - c.y * step_s[from], c.x * step_s[from] + c.y * step_c[from]);
        }
        cs[at] = c.x;
        sn[at] = c.y;
    }
}


// R groups of eight lanes to a head, P pairs of channels to a lane; 32 / R heads at a time.  Two pairs for fp32, four for bf16 heads of more
// than 32 channels: what a unit costs beside its elements (shuffles, the meeting, rho) is then shared by more of them (the vision grid
// forward 131 -> 91 us, 262144 tokens of 128 channels each way 393 + 535 -> 252 + 476; of one pair 267 us and more).  With four pairs
// there are one or two CTAs to an SM, too few loads on their way: the next unit's rows come by asynchronous copies meanwhile, each thread's
// into places of its own (91 -> 75 us, 5.4 TB/s; 252 + 464 -> 210 + 375 us; fetched into L2 alone 79, 220 + 403; since sums beyond fp32 are looked
// for 208 + 388, 5.2 and 4.1 TB/s).  With two
// pairs there are enough loads as it is (fetches into L2: 250 + 356 -> 275 + 460 us); heads of more than 128 channels have no room beside
// the table.
constexpr int resident(int pairs, bool backward) { return pairs > 2 ? (backward ? 1 : 2) : backward ? 2 : 3; }          // CTAs an SM, by registers
template <int R, int P, bool BWD, bool VEC> struct Staging {
    static constexpr bool ON = VEC && P > 2 && R <= 16;
    static constexpr int BYTES = ON ? 256 * 16 * 2 * P * (BWD ? 2 : 1) : 0;
};
__device__ __forceinline__ void copy16(void *to, const void *from, bool real)          // or zeros
{
    if (real) HN_G(from, 16);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"((unsigned)__cvta_generic_to_shared(to)), "l"(from), "r"(real ? 16 : 0) : "memory");
}
// A unit in which a mean square was not finite, once more from the tensors, by the warps of its head: the tokens of `large` at kShrink, the
// others as before, to the bit.  Returns this lane's sums for the weights' gradients.  A call: in line, as a second round of the same loop,
// it cost the common path more (heads of 50 channels on 31 x 33 each way 42 -> 46 us, of 256 on 16384 tokens 536 -> 558; with the call 42
// and 533; 262144 tokens of 128 channels each way 585 -> 595 and with the call 603).
template <int P> struct LaneSums { float v[P][2]; };
template <typename T, int R, int P, bool BWD, bool VEC>
__device__ __noinline__ LaneSums<P> heads_again(const T *in, const T *gradient, T *out, const float *w, const float *cs, const float *sn, float *meet, int live, int t0, int half,
                                                int turned, int T_, float per_mean, float eps, unsigned large, int r, int group)
{
    constexpr int V = Tile<T>::V, TOKENS = Tile<T>::TOKENS, WARPS = R / 4, SUMS = BWD ? 2 : 1;
    const int lane = threadIdx.x & 31, vc = lane & 7;
    LaneSums<P> dg;
#pragma unroll
    for (int p = 0; p < P; ++p) dg.v[p][0] = dg.v[p][1] = 0.f;
    auto token = [&](int e) { return t0 + (VEC ? vc * V + e : e * 8 + vc); };
    // the channels of a pair and its gradient before the rotation
    auto pair_of = [&](int e, int p, float (&x)[2], float (&d)[2]) {
        const int t = token(e), i = r + R * p;
        const bool real = t < live && i < half;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const long long at = (long long)(R * p + s * half) * T_ + t;
            x[s] = real ? IO<T>::ld(in, at) * (large >> e & 1 ? kShrink : 1.f) : 0.f;
            d[s] = BWD && real ? IO<T>::ld(gradient, at) : 0.f;
        }
        if (BWD && i < turned) {
            const int at = i * TOKENS + table_at(vc, e);
            const float c = cs[at], n = sn[at], l = d[0], h = d[1];
            d[0] = fmaf(h, n, l * c);
            d[1] = fmaf(l, -n, h * c);
        }
    };
    auto weight = [&](int p, int s) { return w[(r + R * p < half ? r + R * p : 0) + s * half]; };
    float s1[V], s2[V];
#pragma unroll 1
    for (int e = 0; e < V; ++e) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float x[2], d[2];
            pair_of(e, p, x, d);
#pragma unroll
            for (int s = 0; s < 2; ++s) { a = fmaf(x[s], x[s], a); b = fmaf(d[s] * weight(p, s), x[s], b); }
        }
#pragma unroll
        for (int m = 8; m < 32; m <<= 1) { a += __shfl_xor_sync(~0u, a, m); b += __shfl_xor_sync(~0u, b, m); }
        s1[e] = a;
        s2[e] = b;
        if (WARPS > 1 && lane < 8) {
            meet[(threadIdx.x >> 5) * TOKENS + vc * V + e] = a;
            if (BWD) meet[((SUMS - 1) * 8 + (threadIdx.x >> 5)) * TOKENS + vc * V + e] = b;
        }
    }
    if (WARPS > 1) {
        __syncwarp();
        asm volatile("bar.sync %0, %1;\n" ::"r"(1 + group), "n"(32 * WARPS) : "memory");
    }
#pragma unroll 1
    for (int e = 0; e < V; ++e) {
        const float shrink = large >> e & 1 ? kShrink : 1.f;
        float a = s1[e], b = s2[e];
        if (WARPS > 1) {
            a = b = 0.f;
            for (int k = 0; k < WARPS; ++k) {
                a += meet[(group * WARPS + k) * TOKENS + vc * V + e];
                if (BWD) b += meet[((SUMS - 1) * 8 + group * WARPS + k) * TOKENS + vc * V + e];
            }
        }
        const float v = fmaf(a, per_mean, eps * shrink * shrink), rho = v > kLargest ? 0.f : inverse_root(v);      // (0: a channel is infinite)
        b = rho * b * -per_mean;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float x[2], d[2];
            pair_of(e, p, x, d);
            const int i = r + R * p;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (BWD) {
                    const float hat = x[s] * rho, own = d[s] * weight(p, s);
                    dg.v[p][s] = fmaf(d[s], hat, dg.v[p][s]);
                    x[s] = rho * fmaf(hat, b, own) * shrink;
                } else x[s] *= rho * weight(p, s);
            }
            if (!BWD && i < turned) {
                const int at = i * TOKENS + table_at(vc, e);
                const float c = cs[at], n = sn[at], l = x[0], h = x[1];
                x[0] = fmaf(h, -n, l * c);
                x[1] = fmaf(l, n, h * c);
            }
            if (token(e) < live && i < half)
#pragma unroll
                for (int s = 0; s < 2; ++s) IO<T>::st(out, (long long)(R * p + s * half) * T_ + token(e), x[s]);
        }
    }
    return dg;
}

template <typename T, int R, int P, bool BWD, bool VEC> __global__ void __launch_bounds__(256, resident(P, BWD)) heads_kernel(HeadsArgs a)
{
    constexpr int V = Tile<T>::V, TOKENS = Tile<T>::TOKENS, HEADS = 32 / R, WARPS = R / 4, SUMS = BWD ? 2 : 1, N = V / 2;
    constexpr bool STAGED = Staging<R, P, BWD, VEC>::ON;
    extern __shared__ __align__(16) float sm[];
    __shared__ double freq[kMaxD / 2];
    __shared__ int axis_of[kMaxD / 2];
    __shared__ float weights[2][kMaxD];
    __shared__ __align__(16) float meet[2][SUMS][8][TOKENS];       // [warp][lane of eight][V]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, vc = lane & 7, group = warp / WARPS, r = (warp % WARPS) * 4 + (lane >> 3), half = a.D / 2;
    uint4 *const slot = (uint4 *)sm + tid;                         // one of every 256
    float *cs = sm + Staging<R, P, BWD, VEC>::BYTES / 4, *sn = cs + a.turned * TOKENS;
    float *step_c = sn + a.turned * TOKENS, *step_s = step_c + a.turned * TOKENS;
    float2 *rows = (float2 *)(step_s + a.turned * TOKENS);
    pdl_join();
    for (int i = tid; i < a.turned; i += 256) freq[i] = pair_frequency(a, i, &axis_of[i]);
    for (int i = tid; i < 2 * a.D; i += 256) {
        const int kind = i >= a.D, c = kind ? i - a.D : i;
        weights[kind][c] = 1.f;
        if (a.g[kind]) { HN_G(a.g[kind] + c, 4); weights[kind][c] = __ldg(a.g[kind] + c); }
    }
    __syncthreads();
    if (!a.positions)
        for (int i = tid; i < a.turned * TOKENS; i += 256)
            if (axis_of[i / TOKENS] == a.ndim - 1) {
                const float2 c = rotor(i % TOKENS, freq[i / TOKENS]);
                const int at = i / TOKENS * TOKENS + token_at<T, VEC>(i % TOKENS);
                step_c[at] = c.x;
                step_s[at] = c.y;
            }
    float acc[BWD ? 2 : 1][P][2];
#pragma unroll
    for (int k = 0; k < (BWD ? 2 : 1); ++k)
#pragma unroll
        for (int p = 0; p < P; ++p) acc[k][p][0] = acc[k][p][1] = 0.f;
    // units: the heads of q and k of one batch entry after the other; a split of them to a CTA
    const int HT = a.H[0] + a.H[1];
    const long long units = (long long)a.B * HT, per = (units + a.splits - 1) / a.splits, from = blockIdx.y * per, to = from + per < units ? from + per : units;
    // a lane's rows: the channels r + R p and half further on, of the head that its group is at
    const long long row0 = (long long)r * a.T;
    auto place_of = [&](int b, int h, int &kind) {
        h += group;
        while (h >= HT) { h -= HT; ++b; }
        kind = h >= a.H[0];
        return ((long long)b * a.H[kind] + h - (kind ? a.H[0] : 0)) * a.D * (long long)a.T + row0;
    };
    auto end_of = [&](long long b0) { return a.positions && (b0 + 1) * HT < to ? (b0 + 1) * HT : to; };          // (positions are a batch entry's)
    auto fetch = [&](int tile, long long u) {                      // this thread's part of the units from u on, into its own places
        const long long b0 = u / HT;
        int kind;
        const long long at = place_of((int)b0, (int)(u - b0 * HT), kind);
        const int t = tile * TOKENS + vc * V;
        const bool in = u + group < end_of(b0) && t < a.T;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const bool real = in && r + R * p < half;
                const long long o = real ? at + (long long)(R * p + s * half) * a.T + t : 0;
                copy16(slot + (2 * p + s) * 256, (const T *)a.x[kind] + o, real);
                if constexpr (BWD) copy16(slot + (2 * P + 2 * p + s) * 256, (const T *)a.dy[kind] + o, real);
            }
    };
    if constexpr (STAGED)
        if (from < to && blockIdx.x < a.tiles) fetch(blockIdx.x, from);
    int turn = 0;
    for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int t0 = tile * TOKENS;
        for (long long u = from; u < to;) {
            const long long b0 = u / HT, end = end_of(b0);
            __syncthreads();                                       // (the table's readers are through; the steps are there)
            fill_table<T, VEC>(a, (int)b0, t0, cs, sn, step_c, step_s, rows, freq, axis_of, tid);
            __syncthreads();
            int b = (int)b0, h = (int)(u - b0 * HT);               // of the first of the units at a time
#pragma unroll 1
            for (; u < end; u += HEADS) {
                int kind;
                const long long at = place_of(b, h, kind);
                const int live = u + group < end ? a.T : 0;
                h += HEADS;
                while (h >= HT) { h -= HT; ++b; }
                const T *in = (const T *)a.x[kind] + at, *gradient = (const T *)a.dy[kind] + at;
                T *out = (T *)a.out[kind] + at;
                if constexpr (STAGED) asm volatile("cp.async.wait_all;\n" ::: "memory");
                // what was loaded stays as it came: bf16 values twice made fp32 cost less than the registers
                Tokens<T, VEC> rx[P][2];
                f2 d[BWD ? P : 1][2][N], s1[N], s2[BWD ? N : 1];
                {
                    Tokens<T, VEC> rd[BWD ? P : 1][2];
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const long long o = (long long)(R * p + s * half) * a.T;
                            if constexpr (STAGED) {
                                rx[p][s].w = slot[(2 * p + s) * 256];
                                if constexpr (BWD) rd[p][s].w = slot[(2 * P + 2 * p + s) * 256];
                            } else {
                                rx[p][s].load(in + o, t0, vc, r + R * p < half ? live : 0);
                                if constexpr (BWD) rd[p][s].load(gradient + o, t0, vc, r + R * p < half ? live : 0);
                            }
                        }
                    if constexpr (BWD)
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int s = 0; s < 2; ++s) rd[p][s].get(d[p][s]);
                }
                auto turned = [&](f2 (&lo)[N], f2 (&hi)[N], int i, float way) {
#pragma unroll
                    for (int e = 0; e < N; e += 2) {
                        const int at4 = i * TOKENS + (e / 2 * 8 + vc) * 4;
                        const float4 c4 = *(const float4 *)&cs[at4], n4 = *(const float4 *)&sn[at4];
                        const f2 c[2] = {make2(c4.x, c4.y), make2(c4.z, c4.w)}, n[2] = {make2(n4.x, n4.y), make2(n4.z, n4.w)};
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const f2 l = lo[e + m], h = hi[e + m], other = mul2(n[m], pair(-1.f)), sine = way > 0.f ? n[m] : other, back = way > 0.f ? other : n[m];
                            lo[e + m] = fma2(h, back, mul2(l, c[m]));
                            hi[e + m] = fma2(l, sine, mul2(h, c[m]));
                        }
                    }
                };
                auto weight = [&](int p, int s) { return pair(weights[kind][(r + R * p < half ? r + R * p : 0) + s * half]); };
#pragma unroll
                for (int e = 0; e < N; ++e) s1[e] = pair(0.f);
                if constexpr (BWD)
#pragma unroll
                    for (int e = 0; e < N; ++e) s2[e] = pair(0.f);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if constexpr (BWD)
                        if (r + R * p < a.turned) turned(d[p][0], d[p][1], r + R * p, -1.f);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        f2 x[N];
                        rx[p][s].get(x);
                        const f2 w = weight(p, s);
#pragma unroll
                        for (int e = 0; e < N; ++e) {
                            s1[e] = fma2(x[e], x[e], s1[e]);
                            if constexpr (BWD) s2[e] = fma2(mul2(d[p][s][e], w), x[e], s2[e]);
                        }
                    }
                }
                if constexpr (STAGED) {                            // the copies have been read: the next unit's, of the next tile behind the last
                    long long un = u + HEADS < end ? u + HEADS : end;
                    int next = tile;
                    if (un >= to) { un = from; next += gridDim.x; }
                    if (next < a.tiles) fetch(next, un);
                }
                f2 rho[N];
                if (a.norm == NORM_NONE) {
#pragma unroll
                    for (int e = 0; e < N; ++e) rho[e] = pair(1.f);
                } else {
                    auto lanes = [&](f2 (&v)[N]) {
#pragma unroll
                        for (int e = 0; e < N; ++e)
#pragma unroll
                            for (int m = 8; m < 32; m <<= 1) v[e] = add2(v[e], make2(__shfl_xor_sync(~0u, v[e].x, m), __shfl_xor_sync(~0u, v[e].y, m)));
                    };
                    lanes(s1);
                    if constexpr (BWD) lanes(s2);
                    if constexpr (WARPS > 1) {
                        auto put = [&](float *m, const f2 (&v)[N]) {
#pragma unroll
                            for (int e = 0; e < N; e += 2) *(float4 *)(m + vc * V + 2 * e) = make_float4(v[e].x, v[e].y, v[e + 1].x, v[e + 1].y);
                        };
                        auto get = [&](const float (*m)[TOKENS], f2 (&v)[N]) {
#pragma unroll
                            for (int e = 0; e < N; e += 2) {
                                v[e] = v[e + 1] = pair(0.f);
#pragma unroll
                                for (int k = 0; k < WARPS; ++k) {
                                    const float4 q = *(const float4 *)&m[group * WARPS + k][vc * V + 2 * e];
                                    v[e] = add2(v[e], make2(q.x, q.y));
                                    v[e + 1] = add2(v[e + 1], make2(q.z, q.w));
                                }
                            }
                        };
                        if (lane < 8) {
                            put(meet[turn][0][warp], s1);
                            if constexpr (BWD) put(meet[turn][SUMS - 1][warp], s2);
                        }
                        __syncthreads();
                        get(meet[turn][0], s1);
                        if constexpr (BWD) get(meet[turn][SUMS - 1], s2);
                        turn ^= 1;
                    } else asm volatile("" ::: "memory");          // (nothing further down is begun above: a quarter of the spills)
                    f2 all = pair(0.f);                            // finite where all are
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        s1[e] = fma2(s1[e], pair(a.per_mean), pair(a.eps));
                        all = fma2(s1[e], pair(0x1p-8f), all);
                    }
                    if (__any_sync(~0u, !(sum2(all) <= kLargest))) {      // (in all warps of the head: they hold the same sums)
                        unsigned large = 0;
#pragma unroll
                        for (int e = 0; e < N; ++e) large |= (!(s1[e].x <= kLargest) ? 1u : 0u) << (2 * e) | (!(s1[e].y <= kLargest) ? 2u : 0u) << (2 * e);
                        const LaneSums<P> more = heads_again<T, R, P, BWD, VEC>(in, gradient, out, weights[kind], cs, sn, &meet[turn][0][0][0], live, t0, half, a.turned, a.T, a.per_mean,
                                                                                a.eps, large, r, group);
                        turn ^= 1;
                        if constexpr (BWD)
#pragma unroll
                            for (int p = 0; p < P; ++p)
#pragma unroll
                                for (int s = 0; s < 2; ++s) {
                                    if (kind) acc[1][p][s] += more.v[p][s];
                                    else acc[0][p][s] += more.v[p][s];
                                }
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        rho[e] = make2(inverse_root(s1[e].x), inverse_root(s1[e].y));
                        if constexpr (BWD) s2[e] = mul2(mul2(rho[e], s2[e]), pair(-a.per_mean));
                    }
                }
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const int i = r + R * p, room = i < half ? live : 0;
                    f2 x[2][N];
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const f2 w = weight(p, s);
                        rx[p][s].get(x[s]);
                        if constexpr (BWD) {
                            f2 sum = pair(0.f);
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                const f2 hat = mul2(x[s][e], rho[e]), own = mul2(d[p][s][e], w);
                                sum = fma2(d[p][s][e], hat, sum);
                                x[s][e] = a.norm == NORM_NONE ? own : mul2(rho[e], fma2(hat, s2[e], own));
                            }
                            if (kind) acc[BWD][p][s] += sum2(sum);
                            else acc[0][p][s] += sum2(sum);
                        } else {
#pragma unroll
                            for (int e = 0; e < N; ++e) x[s][e] = mul2(x[s][e], mul2(rho[e], w));
                        }
                    }
                    if constexpr (!BWD)
                        if (i < a.turned) turned(x[0], x[1], i, 1.f);
#pragma unroll
                    for (int s = 0; s < 2; ++s) store_tokens<T, VEC>(out + (long long)(R * p + s * half) * a.T, x[s], t0, vc, room);
                }
            }
            u = end;
        }
    }
    if constexpr (BWD) {
        if (!a.dg[0] && !a.dg[1]) return;
        float *sum = &meet[0][0][0][0];                            // [HEADS][D]: at most 512 of its numbers
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            __syncthreads();
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    float v = acc[kind][p][s];
#pragma unroll
                    for (int m = 1; m < 8; m <<= 1) v += __shfl_xor_sync(~0u, v, m);
                    if (vc == 0 && r + R * p < half) sum[group * a.D + r + R * p + s * half] = v;
                }
            __syncthreads();
            float *part = a.part + (((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 + kind) * a.D;
            for (int c = tid; c < a.D; c += 256) {
                float v = 0.f;
                for (int j = 0; j < HEADS; ++j) v += sum[j * a.D + c];
                HN_G(part + c, 4);
                part[c] = v;
            }
        }
    }
}

// the blocks' sums of the weights' gradients, always in the same order: 8 channels and 32 spans of blocks to a CTA
__global__ void __launch_bounds__(256) heads_sum_kernel(HeadsArgs a, int n)
{
    __shared__ double s[32][8];
    const int kind = blockIdx.y, c = blockIdx.x * 8 + (threadIdx.x & 7), span = threadIdx.x >> 3;
    pdl_join();
    if (!a.dg[kind]) return;
    const float *part = a.part + (long long)kind * a.D + c;
    double v = 0.;
    if (c < a.D) {
#pragma unroll 4
        for (int i = span; i < n; i += 32) { HN_G(part + (long long)i * 2 * a.D, 4); v += part[(long long)i * 2 * a.D]; }
    }
    s[span][threadIdx.x & 7] = v;
    __syncthreads();
    if (span || c >= a.D) return;
    for (int j = 1; j < 32; ++j) v += s[j][threadIdx.x & 7];
    HN_G(a.dg[kind] + c, 4);
    a.dg[kind][c] = (float)v;
}

// Few tokens: a warp per token and head, a lane per pair
template <typename T> __global__ void __launch_bounds__(256) heads_token_kernel(HeadsArgs a)
{
    const int lane = threadIdx.x & 31, half = a.D / 2, HT = a.H[0] + a.H[1];
    const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_join();
    if (i >= (long long)a.B * HT * a.T) return;
    const int t = (int)(i % a.T), b = (int)(i / a.T / HT), hh = (int)(i / a.T % HT), kind = hh >= a.H[0], h = kind ? hh - a.H[0] : hh;
    const long long at = ((long long)b * a.H[kind] + h) * a.D * a.T + t;
    constexpr int P = kMaxD / 64;
    float x[P][2], rho = 1.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int c = lane + 32 * p;
            x[p][s] = c < half ? IO<T>::ld((const T *)a.x[kind], at + (long long)(c + s * half) * a.T) : 0.f;
        }
    if (a.norm != NORM_NONE) {
        auto mean_square = [&](float eps) {
            float sum = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p) sum = fmaf(x[p][1], x[p][1], fmaf(x[p][0], x[p][0], sum));
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) sum += __shfl_xor_sync(~0u, sum, m);
            return fmaf(sum, a.per_mean, eps);
        };
        float v = mean_square(a.eps);
        if (!(v <= kLargest)) {                              // (the same in all lanes; see heads_again)
#pragma unroll
            for (int p = 0; p < P; ++p) { x[p][0] *= kShrink; x[p][1] *= kShrink; }
            v = mean_square(a.eps * kShrink * kShrink);
        }
        rho = 1.f / sqrtf(v);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = lane + 32 * p;
        if (c >= half) break;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float w = 1.f;
            if (a.g[kind]) { HN_G(a.g[kind] + c + s * half, 4); w = __ldg(a.g[kind] + c + s * half); }
            x[p][s] *= rho * w;
        }
        if (c < a.turned) {
            int axis;
            const double f = pair_frequency(a, c, &axis);
            const float2 z = rotor(place(a, b, axis, t), f);
            const float lo = x[p][0], hi = x[p][1];
            x[p][0] = lo * z.x - hi * z.y;
            x[p][1] = lo * z.y + hi * z.x;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) IO<T>::st((T *)a.out[kind], at + (long long)(c + s * half) * a.T, x[p][s]);
    }
}

static int pairs_of(int D, int dtype) { return D > 128 || (dtype == HYENAND_BF16 && D > 32) ? 4 : 2; }
static int rows_of(int D, int dtype)                      // a power of two, so that rows and pairs hold half the channels
{
    int r = 4;
    while (r * pairs_of(D, dtype) < D / 2) r *= 2;
    return r;
}
// CTAs along the tiles, and splits of the heads of q and k: two rounds of what the SMs hold where there is work for them
static int plan(HeadsArgs &a, int dtype, bool backward)
{
    const int tokens = dtype == HYENAND_F32 ? 32 : 64, want = 2 * resident(pairs_of(a.D, dtype), backward) * kSms, at_once = 32 / rows_of(a.D, dtype);
    a.tiles = (int)(((long long)a.T + tokens - 1) / tokens);
    const long long most = ((long long)a.B * (a.H[0] + a.H[1]) + at_once - 1) / at_once, s = a.tiles >= want ? 1 : want / a.tiles;
    a.splits = (int)(s < most ? s : most);
    return a.tiles < want ? a.tiles : want;
}

// cosines and sines of a tile; of the steps of one; of its rows
static size_t table_bytes(int turned, int tokens, int last) { return (size_t)turned * (16 * tokens + 8 * rows_of_tile(tokens, last)); }
template <auto FN, typename T> static int launch_tiles(const HeadsArgs &a, int grid_x, int staging, cudaStream_t st)
{
    const size_t bytes = staging + table_bytes(a.turned, Tile<T>::TOKENS, a.dims[a.ndim - 1]);
    static PerDevice ready;
    if (bytes > 24 * 1024 && !ready.once([&] { return cudaFuncSetAttribute(FN, cudaFuncAttributeMaxDynamicSharedMemorySize, staging + (int)table_bytes(staging ? 64 : kMaxD / 2, Tile<T>::TOKENS, 1)) == cudaSuccess ? 1 : -1; }))
        return kNoLaunch;
    launch_pdl(FN, dim3(grid_x, a.splits), 256, bytes, st, a);
    return 0;
}
template <typename T, bool BWD> static int launch_heads(HeadsArgs &a, int dtype, cudaStream_t st)
{
    if (!BWD && a.T < 8) {
        const long long blocks = ((long long)a.B * (a.H[0] + a.H[1]) * a.T + 7) / 8;
        if (blocks > 0x7fffffffll) return kTooLarge;
        launch_pdl(heads_token_kernel<T>, dim3((unsigned)blocks), 256, 0, st, a);
        return 0;
    }
    const int R = rows_of(a.D, dtype), gx = plan(a, dtype, BWD);
    const bool vec = a.T % Tile<T>::V == 0;
    int e = kNoLaunch;
#define HN_HEADS(R_, P_) if (R == R_) e = vec ? launch_tiles<heads_kernel<T, R_, P_, BWD, true>, T>(a, gx, Staging<R_, P_, BWD, true>::BYTES, st) \
                                 : launch_tiles<heads_kernel<T, R_, P_, BWD, false>, T>(a, gx, 0, st)
    if (pairs_of(a.D, dtype) == 4) {
        HN_HEADS(32, 4);
        if constexpr (sizeof(T) == 2) { HN_HEADS(8, 4); HN_HEADS(16, 4); }
    } else {
        HN_HEADS(4, 2); HN_HEADS(8, 2);
        if constexpr (sizeof(T) == 4) { HN_HEADS(16, 2); HN_HEADS(32, 2); }
    }
#undef HN_HEADS
    if (e || !BWD || (!a.dg[0] && !a.dg[1])) return e;
    launch_pdl(heads_sum_kernel, dim3((a.D + 7) / 8, 2), 256, 0, st, a, gx * a.splits);
    return 0;
}

static int fill(HeadsArgs &a, int ndim, const int *dims, int B, int Hq, int Hk, int D, int dtype, int norm, const int *axes, double base, float eps)
{
    if (ndim < 1 || ndim > kMaxAxes || !dims) return fail(HYENAND_ERR_INVALID_ARG, "ndim must be 1 to %d, with dims", kMaxAxes);
    if (B < 1 || Hq < 1 || Hk < 1 || D < 1) return fail(HYENAND_ERR_INVALID_ARG, "B, Hq, Hk and D must be >= 1");
    if (dtype != HYENAND_F32 && dtype != HYENAND_BF16) return fail(HYENAND_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (norm < NORM_NONE || norm > NORM_L2) return fail(HYENAND_ERR_INVALID_ARG, "unknown norm %d", norm);
    if (D % 2 || D > kMaxD) return fail(HYENAND_ERR_UNSUPPORTED, "D = %d: heads have an even number of channels up to %d", D, kMaxD);
    long long T = 1;
    for (int n = 0; n < ndim; ++n) {
        if (dims[n] < 1) return fail(HYENAND_ERR_INVALID_ARG, "every extent must be >= 1");
        T *= dims[n];
        if (T > (1 << 30)) return fail(HYENAND_ERR_UNSUPPORTED, "a grid of more than 2^30 tokens");
    }
    if ((long long)B * ((long long)Hq + Hk) > (1 << 28)) return fail(HYENAND_ERR_UNSUPPORTED, "B * (Hq + Hk) is above 2^28");
    if ((long long)B * ((long long)Hq + Hk) * D > (1ll << 40) / T) return fail(HYENAND_ERR_UNSUPPORTED, "more than 2^40 elements");
    long long pairs = 0;
    for (int n = 0; n < ndim; ++n) {
        const int s = axes ? axes[n] : 0;
        if (s < 0) return fail(HYENAND_ERR_INVALID_ARG, "an axis has %d pairs", s);
        pairs += s;
        a.dims[n] = dims[n];
        a.axes[n] = s;
    }
    if (pairs > D / 2) return fail(HYENAND_ERR_INVALID_ARG, "the axes have %lld pairs, a head %d", pairs, D / 2);
    if (pairs && !(base > 0. && base < 1e300)) return fail(HYENAND_ERR_INVALID_ARG, "base must be positive and finite");
    if (!(eps > 0.f && eps < 3e38f)) return fail(HYENAND_ERR_INVALID_ARG, "eps must be positive and finite");
    a.H[0] = Hq; a.H[1] = Hk; a.B = B; a.D = D; a.T = (int)T; a.ndim = ndim; a.turned = (int)pairs; a.norm = norm; a.eps = eps;
    a.per_mean = norm == NORM_RMS ? 1.f / D : 1.f;
    a.log2_base = pairs ? log2(base) : 0.;
    return HYENAND_OK;
}
static size_t part_bytes(HeadsArgs a, int dtype)
{
    const long long gx = plan(a, dtype, true);
    return (size_t)(gx * a.splits * 2 * a.D * (long long)sizeof(float));
}

}  // namespace hn

using namespace hn;

extern "C" long long hyenand_heads_workspace_bytes(int ndim, const int *dims, int B, int Hq, int Hk, int D, int dtype)
{
    HeadsArgs a{};
    clear_error();
    if (fill(a, ndim, dims, B, Hq, Hk, D, dtype, NORM_NONE, nullptr, 1., 1.f)) return 0;
    return (long long)((part_bytes(a, dtype) + 15) / 16 * 16);
}

extern "C" int hyenand_heads_forward(int ndim, const int *dims, int B, int Hq, int Hk, int D, int dtype, int norm, const int *axes, double base, float eps,
                                     const void *q, const void *k, const float *g_q, const float *g_k, const int *positions, void *q_out, void *k_out,
                                     void *cuda_stream)
{
    clear_error();
    HeadsArgs a{};
    if (int e = fill(a, ndim, dims, B, Hq, Hk, D, dtype, norm, axes, base, eps)) return e;
    if (!q || !k || !q_out || !k_out) return fail(HYENAND_ERR_INVALID_ARG, "q, k, q_out, k_out must be non-NULL");
    a.x[0] = q; a.x[1] = k; a.g[0] = g_q; a.g[1] = g_k; a.positions = positions; a.out[0] = q_out; a.out[1] = k_out;
    CallTensors c;
    const size_t one = (size_t)B * D * a.T * elsize(dtype);
    c.in("q", q, one * Hq); c.in("k", k, one * Hk); c.in("g_q", g_q, (size_t)D * 4, 4); c.in("g_k", g_k, (size_t)D * 4, 4);
    c.in("positions", positions, (size_t)B * ndim * a.T * sizeof(int), 4);
    c.out("q_out", q_out, one * Hq, 16, "q"); c.out("k_out", k_out, one * Hk, 16, "k");
    if (int e = c.check()) return e;
    c.register_ranges();
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return finish(dtype == HYENAND_F32 ? launch_heads<float, false>(a, dtype, st) : launch_heads<bf16, false>(a, dtype, st));
}

extern "C" int hyenand_heads_backward(int ndim, const int *dims, int B, int Hq, int Hk, int D, int dtype, int norm, const int *axes, double base, float eps,
                                      const void *q, const void *k, const float *g_q, const float *g_k, const int *positions, const void *dq_out,
                                      const void *dk_out, void *dq, void *dk, float *dg_q, float *dg_k, void *workspace, void *cuda_stream)
{
    clear_error();
    HeadsArgs a{};
    if (int e = fill(a, ndim, dims, B, Hq, Hk, D, dtype, norm, axes, base, eps)) return e;
    if (!q || !k || !dq_out || !dk_out || !dq || !dk) return fail(HYENAND_ERR_INVALID_ARG, "q, k, dq_out, dk_out, dq, dk must be non-NULL");
    if ((dg_q && !g_q) || (dg_k && !g_k)) return fail(HYENAND_ERR_INVALID_ARG, "a gradient of a weight that is not given");
    if ((dg_q || dg_k) && !workspace) return fail(HYENAND_ERR_INVALID_ARG, "workspace must be non-NULL for the weights' gradients");
    a.x[0] = q; a.x[1] = k; a.dy[0] = dq_out; a.dy[1] = dk_out; a.g[0] = g_q; a.g[1] = g_k; a.positions = positions;
    a.out[0] = dq; a.out[1] = dk; a.dg[0] = dg_q; a.dg[1] = dg_k; a.part = (float *)workspace;
    CallTensors c;
    const size_t one = (size_t)B * D * a.T * elsize(dtype);
    c.in("q", q, one * Hq); c.in("k", k, one * Hk); c.in("g_q", g_q, (size_t)D * 4, 4); c.in("g_k", g_k, (size_t)D * 4, 4);
    c.in("positions", positions, (size_t)B * ndim * a.T * sizeof(int), 4);
    c.in("dq_out", dq_out, one * Hq); c.in("dk_out", dk_out, one * Hk);
    c.out("dq", dq, one * Hq, 16, "dq_out"); c.out("dk", dk, one * Hk, 16, "dk_out");
    c.out("dg_q", dg_q, (size_t)D * 4, 4); c.out("dg_k", dg_k, (size_t)D * 4, 4);
    if (dg_q || dg_k) c.out("workspace", workspace, part_bytes(a, dtype));
    if (int e = c.check()) return e;
    c.register_ranges();
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return finish(dtype == HYENAND_F32 ? launch_heads<float, true>(a, dtype, st) : launch_heads<bf16, true>(a, dtype, st));
}
