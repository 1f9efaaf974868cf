// The gated linear recurrence along the last axis, forward, backward and for one token:
//
//     s_t = a_t s_{t-1} + k_t v_t,      y_t = q_t s_t,      a_t = g_t | exp(g_t) | sigmoid(g_t)
//
// One pass over the data.  Maps s -> A s + S of neighbouring positions compose to (A1 A2, S2 + A2 S1); a thread composes those of its
// positions, the lanes of a row scan the threads' by shuffles, the warps of a row meet in shared memory, and then every thread runs
// its steps from the state that enters them.  Long rows are walked tile by tile, the state carried on.  Rows too few to fill the GPU
// are cut into segments: a first kernel leaves every segment's map in the workspace, the second composes those in front of its own.
//
// All states and maps are fp32.  A product of thousands of decays close to 1 would collect the rounding of each of them, always to
// the same side where the decay is constant; the maps therefore carry P = A - 1 beside A (P1 P2 + P1 + P2), built from 1 - a_t
// (sigmoid), from the sum of the g_t (exp), and use whichever of the two is the precise one.
#include <atomic>

#include "entry.cuh"
#include "octet.cuh"
#include "pair.cuh"
#include "tma_util.cuh"

namespace hn {

constexpr int kMarkOctets = 32;           // the state is marked in front of every 256 positions of a row (octets of the flat tensor)

enum { DECAY_VALUE = 0, DECAY_LOG = 1, DECAY_SIGMOID = 2 };

struct RecArgs {
    const void *q, *k, *v, *g, *dy;
    const float *s0, *ds_end;             // [rows] or nullptr: zero
    const int *lengths;                   // [B] or nullptr: L
    void *y, *dq, *dk, *dv, *dg;
    float *s_end, *ds0;                   // [rows] or nullptr
    float *marks;                         // [rows][marks_row] or nullptr (forward); read by the backward
    float4 *maps;                         // [rows][segments], where there are several (Row::way_end)
    int segments;                         // of a row
    long long rows, n;                    // n = rows * L
    int C, L, marks_row;
#ifdef HYENAND_DEBUG
    int late_tile, late_warp;             // whose copies are taken to come too late: of every row (-1: none), of a CTA (-1: all)
#endif
};
#ifdef HYENAND_DEBUG
static __device__ __forceinline__ bool is_late(const RecArgs &p, int tile) { return p.late_tile == tile && (p.late_warp < 0 || p.late_warp == (int)threadIdx.x / 32); }
#else
static __device__ __forceinline__ bool is_late(const RecArgs &, int) { return false; }
#endif

static __device__ int hn_rec_status;                         // 1: a bounded wait gave up

struct Map { float A, P, S; };            // s -> (1 + P) s + S, A = 1 + P
__device__ __forceinline__ float apply(const Map &m, float s)
{
    const bool small = m.A < 0.5f;
    return fmaf(small ? m.A : m.P, s, small ? 0.f : s) + m.S;
}
// a first, then b
__device__ __forceinline__ Map compose(const Map &a, const Map &b) { return {a.A * b.A, fmaf(a.P, b.P, a.P + b.P), apply(b, a.S)}; }

// a_t and 1 - a_t (LOG: see decays).  The approximate exponential and reciprocal are off by a few roundings, which a thread's steps
// can multiply up sixteen-fold at most: what goes on from thread to thread is built from 1 - a_t and the sum of the g_t.
constexpr float kLog2e = 1.4426950408889634f;
template <int DECAY> __device__ __forceinline__ void decay(float g, float &a, float &na)
{
    if constexpr (DECAY == DECAY_VALUE) { a = g; na = 1.f - g; }
    else {
        static_assert(DECAY == DECAY_SIGMOID, "");
        // the larger one as 1 - the smaller: half a unit off, to no side, where the reciprocal's 1 / (1 + e) drifted by 5e-7 of a state over a
        // thread's steps
        const float e = ex2(-kLog2e * fabsf(g)), x = e * rcp(1.f + e), r = 1.f - x;
        a = g >= 0.f ? r : x;
        na = g >= 0.f ? x : r;
    }
}

// exp(x) - 1, given exp(x): the series where they are close to 0 and 1 (its first term left out is below 2^-24 of it)
__device__ __forceinline__ float expm1_of(float x, float ex)
{
    float p = 1.f / 40320.f;
    p = fmaf(p, x, 1.f / 5040.f); p = fmaf(p, x, 1.f / 720.f); p = fmaf(p, x, 1.f / 120.f); p = fmaf(p, x, 1.f / 24.f);
    p = fmaf(p, x, 1.f / 6.f); p = fmaf(p, x, 0.5f); p = fmaf(p, x, 1.f);
    return fabsf(x) < 0.5f ? p * x : ex - 1.f;
}

// a and 1 - a of a thread's positions, and A, P of the whole.  Positions outside [lo, hi) are the identity: their gate is made one
// that decays nothing before anything is computed (whatever was in them).
template <int DECAY, int N> __device__ __forceinline__ void decays(const f2 (&g)[N], f2 (&a)[N], f2 (&na)[N], float &A, float &P)
{
    A = 1.f; P = 0.f;
    if constexpr (DECAY == DECAY_LOG) {
        f2 sum = pair(0.f);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const f2 y = mul2(g[e], pair(kLog2e));
            a[e] = make2(ex2(y.x), ex2(y.y));
            sum = add2(sum, g[e]);
        }
        const float x = sum2(sum);
        A = ex2(x * kLog2e);
        P = expm1_of(x, A);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            decay<DECAY>(g[e].x, a[e].x, na[e].x);
            decay<DECAY>(g[e].y, a[e].y, na[e].y);
            A *= a[e].x * a[e].y;
            P = fmaf(fmaf(P, a[e].x, -na[e].x), a[e].y, -na[e].y);
        }
    }
}
template <int DECAY> __device__ __forceinline__ float no_decay() { return DECAY == DECAY_VALUE ? 1.f : DECAY == DECAY_LOG ? 0.f : __int_as_float(0x7f800000); }
template <int N> __device__ __forceinline__ void mask(f2 (&f)[N], int lo, int hi, float with)
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (2 * e < lo || 2 * e >= hi) f[e].x = with;
        if (2 * e + 1 < lo || 2 * e + 1 >= hi) f[e].y = with;
    }
}

// inclusive scan over the LANES lanes of a row towards higher (UP) or lower lanes
template <int LANES, bool UP> __device__ __forceinline__ Map scan_lanes(Map m, int lane)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
        Map o;
        o.A = UP ? __shfl_up_sync(~0u, m.A, d, LANES) : __shfl_down_sync(~0u, m.A, d, LANES);
        o.P = UP ? __shfl_up_sync(~0u, m.P, d, LANES) : __shfl_down_sync(~0u, m.P, d, LANES);
        o.S = UP ? __shfl_up_sync(~0u, m.S, d, LANES) : __shfl_down_sync(~0u, m.S, d, LANES);
        if (UP ? lane >= d : lane + d < LANES) m = compose(o, m);
    }
    return m;
}
template <int LANES, bool UP> __device__ __forceinline__ Map neighbour(const Map &m, int lane)
{
    Map o;
    o.A = UP ? __shfl_up_sync(~0u, m.A, 1, LANES) : __shfl_down_sync(~0u, m.A, 1, LANES);
    o.P = UP ? __shfl_up_sync(~0u, m.P, 1, LANES) : __shfl_down_sync(~0u, m.P, 1, LANES);
    o.S = UP ? __shfl_up_sync(~0u, m.S, 1, LANES) : __shfl_down_sync(~0u, m.S, 1, LANES);
    if (UP ? lane == 0 : lane == LANES - 1) o = {1.f, 0.f, 0.f};
    return o;
}

// Where a thread stands: LANES lanes share a row (a part of a warp, or a CTA of LANES threads).  A thread takes one octet, or in longer
// rows of bf16 two (OCT): what a tile costs besides its elements (the scans, half of all instructions with one octet) is then a
// smaller part of what the memory allows.
template <int LANES> struct RowLane {
    static constexpr int kThreads = LANES <= 32 ? 128 : LANES;
    static constexpr int kRows = LANES <= 32 ? kThreads / LANES : 1;
    static constexpr int kWarps = LANES <= 32 ? 1 : LANES / 32;      // of one CTA, that share a row
};

// How the warps of a row learn the state that enters them: each leaves its map, the thread that forms the state behind a tile leaves
// that.  A slot is written again two tiles later, when all have passed the barrier of the tile between.
template <int LANES> struct alignas(16) Meeting {
    float4 warp[2][RowLane<LANES>::kWarps];
    float carry[2];
};
template <int LANES, bool UP> struct Step {                   // one thread's part of a tile
    static constexpr int W = LANES < 32 ? LANES : 32, NW = RowLane<LANES>::kWarps;
    Map before;                                              // the positions of the warp in front of this thread's
    Map all;                                                 // those of the whole warp (LANES <= 32: of the row)
    __device__ __forceinline__ explicit Step(const Map &own)
    {
        const int lane = threadIdx.x % W;
        constexpr int last = UP ? W - 1 : 0;
        const Map inc = scan_lanes<W, UP>(own, lane);
        before = neighbour<W, UP>(inc, lane);
        if constexpr (LANES <= 32) all = {__shfl_sync(~0u, inc.A, last, W), __shfl_sync(~0u, inc.P, last, W), __shfl_sync(~0u, inc.S, last, W)};
        else all = inc;                                      // (the last lane's)
    }
    // before the CTA's barrier
    __device__ __forceinline__ void leave(Meeting<LANES> &m, int count) const
    {
        if (LANES > 32 && threadIdx.x % 32 == (UP ? 31 : 0)) m.warp[count & 1][threadIdx.x / 32] = make_float4(all.A, all.P, all.S, 0.f);
    }
    // After it: the state in front of this thread's positions, from the one in front of the tile.  LANES <= 32: carry moves on to the
    // one behind it; else the thread that forms that one stores it (Meeting::carry).
    __device__ __forceinline__ float enter(const Meeting<LANES> &m, int count, float &carry) const
    {
        if constexpr (LANES <= 32) {
            const float s = apply(before, carry);
            carry = apply(all, carry);
            return s;
        } else {
            float in = carry;
            const int w = threadIdx.x / 32;
#pragma unroll
            for (int i = 0; i < NW - 1; ++i) {
                if (i >= (UP ? w : NW - 1 - w)) break;
                const float4 f = m.warp[count & 1][UP ? i : NW - 1 - i];
                in = apply({f.x, f.y, f.z}, in);
            }
            return apply(before, in);
        }
    }
};

// A row, or a segment of one, as its threads see it.
template <int LANES, int E> struct Row {
    using R = RowLane<LANES>;
    static constexpr int kTile = E * LANES;
    long long row, start;                                    // start: its first element
    int l, lead, len;                                        // this thread of a tile; elements of the row's first octet in front of it
    int segment, first, last, live;                          // tiles [first, last) of the row; those below `live` have a position
    bool real;
    __device__ __forceinline__ explicit Row(const RecArgs &p)
    {
        row = (long long)(blockIdx.x / p.segments) * R::kRows + threadIdx.x / LANES;
        segment = (int)(blockIdx.x % p.segments);
        real = row < p.rows;
        l = threadIdx.x % LANES;
        len = real ? p.L : 0;
        if (real && p.lengths) {
            const int b = (int)(row / p.C);
            HN_G(p.lengths + b, 4);
            len = max(0, min(p.L, __ldg(p.lengths + b)));
        }
        start = real ? row * p.L : 0;
        lead = (int)(start & 7);
        const int tiles = (lead + p.L + kTile - 1) / kTile, each = (tiles + p.segments - 1) / p.segments;
        first = min(tiles, segment * each);
        last = min(tiles, first + each);
        live = len ? (lead + len + kTile - 1) / kTile : 0;
    }
    __device__ __forceinline__ int position(int tile) const { return (tile * LANES + l) * E - lead; }           // this thread's first
    __device__ __forceinline__ int warp_position(int tile) const { return (tile * LANES + l - ((int)threadIdx.x & 31)) * E - lead; }
    // Where the way through the segments ends; nothing needs that one's map, its place holds the state that the way begins with
    // (s0 and s_end may be one tensor, and the segments of a row run in any order).
    template <bool UP> __device__ __forceinline__ int way_end(const RecArgs &p) const { return UP ? p.segments - 1 : 0; }
    // by the lanes of one warp: from that state through the segments on the way to this one
    template <bool UP> __device__ __forceinline__ float entering(const RecArgs &p) const
    {
        float state = 0.f;
        if (real) {
            const float4 *f = p.maps + row * p.segments + way_end<UP>(p);
            HN_G(f, 16);
            state = f->z;
        }
        const int lane = threadIdx.x & 31, each = ((UP ? segment : p.segments - 1 - segment) + 31) / 32;
        int n = UP ? segment : p.segments - 1 - segment;
        if (!real) n = 0;
        Map m = {1.f, 0.f, 0.f};
        const int end = min(n, (lane + 1) * each);
        for (int i = lane * each; i < end; i += 8) {
            float4 w[8];                                     // (on their way together)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                w[u] = make_float4(1.f, 0.f, 0.f, 0.f);
                if (i + u < end) {
                    const float4 *f = p.maps + row * p.segments + (UP ? i + u : p.segments - 1 - i - u);
                    HN_G(f, 16);
                    w[u] = *f;
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u < end) m = compose(m, {w[u].x, w[u].y, w[u].z});
        }
        m = scan_lanes<32, true>(m, lane);
        return __shfl_sync(~0u, apply(m, state), 31);
    }
};

// A thread's positions.  Rows of several tiles and of two octets a thread (STAGED) pass through shared memory, 32 bytes a thread and
// tensor: a warp's 1024 of the next tile travel in as one bulk copy a tensor while this tile is worked on, results go out the same way.
// (As 16-byte copies, each lane its own two: 404 and 697 us for 512 rows of 262144, bf16; neighbouring lanes neighbouring pieces:
// 514 and 657, the addresses and conditions of sixteen copies being most of the instructions.)  Every warp has its own barriers.
// A wait for copies is bounded.  A warp whose wait gives up fetches and stores nothing more, and its map is NaN for those who go on
// from there; what was still on its way gets the same time once more to land before the warp leaves, so that nothing reaches shared
// memory that is another CTA's by then.  (Where that second wait stands is the faster of two ways: behind the row forward, 512 rows of
// 262144 242 us and 244 at once; at once backward, 250 rows of 262144 269 and 279 behind the row.)
template <typename T, int OCT, int TENSORS, int THREADS, bool STAGED> struct Places {
    static constexpr int E = 8 * OCT, STAGE = STAGED ? TENSORS * THREADS * 32 : 0;
    static constexpr unsigned WARP_BYTES = 1024;
    static_assert(!STAGED || E * sizeof(T) == 32, "32 bytes a thread");
    const T *in[TENSORS];
    char *mine;                                              // this thread's place of tensor 0 in stage 0
    uint64_t *bars;                                          // this warp's two, and behind them the tile at which a wait gave up
    long long n;
    int len, lane;
    float none;                                              // 0; NaN once a wait has given up (the same in all lanes)

    __device__ __forceinline__ char *place(int turn, int tensor) const { return mine + turn * STAGE + tensor * THREADS * 32; }
    __device__ __forceinline__ void init(char *stages, uint64_t *barriers, int row_len, long long elements)
    {
        mine = stages + threadIdx.x * 32; bars = barriers + 3 * (threadIdx.x / 32); lane = threadIdx.x & 31;
        len = row_len; n = elements; none = 0.f;
        if (STAGED && lane == 0) { mbar_init(bars, 1); mbar_init(bars + 1, 1); fence_mbar_init(); }
        __syncwarp();
    }
    // the positions of this warp, whose first is t of its row and element i of the tensor; by all its lanes.  Nothing is in the way: the
    // lanes have read what was in this stage, and results that left from it have been read by their copies
    __device__ __forceinline__ void fetch(int turn, long long i, int t) const
    {
        if (t + 32 * E <= len) {                             // (what one lane does counts as much as what 32 do: few instructions here)
            if (lane == 0) {
                mbar_expect_tx(bars + turn, TENSORS * WARP_BYTES);
#pragma unroll
                for (int k = 0; k < TENSORS; ++k) { HN_G(in[k] + i, WARP_BYTES); bulk_load(place(turn, k), in[k] + i, WARP_BYTES, bars + turn); }
            }
            return;
        }
        if (t >= len) return;
        const long long last = i + min(32 * E, (len - t + 7) & ~7), end = last <= n ? last : n & ~7ll;        // whole octets of the tensor
        if (lane == 0) {
            const unsigned bytes = (unsigned)(end - i) * (unsigned)sizeof(T);
            mbar_expect_tx(bars + turn, TENSORS * bytes);
            if (bytes)
                for (int k = 0; k < TENSORS; ++k) { HN_G(in[k] + i, bytes); bulk_load(place(turn, k), in[k] + i, bytes, bars + turn); }
        }
        if (last > n && end + lane < n) {                    // (the octet that the tensor ends in)
            for (int k = 0; k < TENSORS; ++k) {
                HN_G(in[k] + end + lane, sizeof(T));
                reinterpret_cast<T *>(place(turn, k) - lane * 32)[end - i + lane] = in[k][end + lane];
            }
            fence_async_smem();                              // (rows walked from the end have copies land in this stage later; the warp meets
                                                             // once more before it reads the octet)
        }
    }
    __device__ __forceinline__ bool good() const { return !STAGED || none == 0.f; }
    __device__ __forceinline__ void drain(int turn, int phase, int t) const { if (t < len) mbar_wait(bars + turn, phase); }
    // All lanes alike; whether the copies of this tile (positions from t on) are here.  Where it first says no, the caller drains.
    __device__ __forceinline__ bool wait(int turn, int phase, int t, bool hold)
    {
        bool here = true;
        if (t < len && good()) here = !hold && mbar_wait(bars + turn, phase);
        if (!__any_sync(~0u, !here)) return true;
        none = __int_as_float(0x7fffffff);
        return false;
    }
    __device__ __forceinline__ void keep_late(int tile) const { if (lane == 0) bars[2] = (uint64_t)tile; }
    __device__ __forceinline__ int late() const { __syncwarp(); return (int)bars[2]; }
    // this thread's positions, the first at element i
    __device__ __forceinline__ void get(int turn, int tensor, long long i, f2 (&f)[E / 2]) const
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int o = 0; o < OCT; ++o) {
                uint4 w;
                if constexpr (STAGED) w = reinterpret_cast<const uint4 *>(place(turn, tensor))[o];
                else { Octet<T> x; x.ld(in[tensor], i, n); w = x.w; }
                f[4 * o] = widen2(w.x); f[4 * o + 1] = widen2(w.y); f[4 * o + 2] = widen2(w.z); f[4 * o + 3] = widen2(w.w);
            }
        } else {
            float4 a, b;
            if constexpr (STAGED) { a = reinterpret_cast<const float4 *>(place(turn, tensor))[0]; b = reinterpret_cast<const float4 *>(place(turn, tensor))[1]; }
            else { Octet<T> x; x.ld(in[tensor], i, n); a = x.a; b = x.b; }
            f[0] = make2(a.x, a.y); f[1] = make2(a.z, a.w); f[2] = make2(b.x, b.y); f[3] = make2(b.z, b.w);
        }
    }
    // Results of the row's L positions; by all lanes of a warp at once, through the place of a tensor that nobody reads any more.
    // t, i: as in fetch; t0, i0: this thread's first
    __device__ __forceinline__ void put(int turn, int tensor, T *p, long long i, int t, long long i0, int t0, int L, const f2 (&f)[E / 2]) const
    {
        if constexpr (!STAGED) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) split2(f[e], x[2 * e], x[2 * e + 1]);
            if (t0 < L && t0 > -8) st_octet(p, i0, max(0, -t0), min(8, L - t0), x);
        } else {
            uint4 *to = reinterpret_cast<uint4 *>(place(turn, tensor));
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                if constexpr (sizeof(T) == 2) to[o] = make_uint4(narrow2(f[4 * o]), narrow2(f[4 * o + 1]), narrow2(f[4 * o + 2]), narrow2(f[4 * o + 3]));
                else reinterpret_cast<float4 *>(to)[o] = make_float4(f[2 * o].x, f[2 * o].y, f[2 * o + 1].x, f[2 * o + 1].y);
            }
            fence_async_smem();
            __syncwarp();
            if (t >= 0 && t + 32 * E <= L) {
                if (lane == 0) { HN_G(p + i, WARP_BYTES); bulk_store(p + i, place(turn, tensor), WARP_BYTES); }
                return;
            }
            const int from = t < 0 ? 8 : 0, whole = min(32 * E, (L - t) & ~7);         // octets that are the row's alone
            if (lane == 0 && whole > from) {
                HN_G(p + i + from, (whole - from) * sizeof(T));
                bulk_store(p + i + from, place(turn, tensor) + from * sizeof(T), (whole - from) * sizeof(T));
            }
            // the octets that it shares with its neighbours
            const T *base = reinterpret_cast<const T *>(place(turn, tensor) - lane * 32);
            if (t < 0 && lane < 8 && t + lane >= 0 && t + lane < L) { HN_G(p + i + lane, sizeof(T)); p[i + lane] = base[lane]; }
            const int rest = max(whole, from);
            if (rest < 32 * E && t + rest + lane < L && lane < 8) { HN_G(p + i + rest + lane, sizeof(T)); p[i + rest + lane] = base[rest + lane]; }
        }
    }
    __device__ __forceinline__ void put_done() const { if (STAGED && lane == 0) tma_commit(); }           // behind a tile's results
    __device__ __forceinline__ void stage_free() const                                              // the last tile's results have left
    {
        if (STAGED && lane == 0) tma_wait_read0();
        __syncwarp();
    }
};

// The map of every segment: of the states (UP, from k, v, g) or of their gradients (from q, dy, g, from the end).
template <typename T, int DECAY, int OCT, bool UP>
__global__ void __launch_bounds__(128, 8) recurrence_maps_kernel(RecArgs p)
{
    constexpr int LANES = 32;
    constexpr int E = 8 * OCT, N = E / 2;
    using Pl = Places<T, OCT, 3, 128, true>;
    extern __shared__ __align__(16) char stages[];
    __shared__ uint64_t barriers[3 * 128 / 32];
    pdl_join();
    const Row<LANES, E> r(p);
    Pl pl;
    pl.in[0] = (const T *)(UP ? p.k : p.q); pl.in[1] = (const T *)(UP ? p.v : p.dy); pl.in[2] = (const T *)p.g;
    pl.init(stages, barriers, r.len, p.n);
    const bool end = r.segment == r.template way_end<UP>(p);
    const int tiles = end ? 0 : max(0, min(r.last, r.live) - r.first);
    auto tile_of = [&](int c) { return UP ? r.first + c : r.first + tiles - 1 - c; };
    auto fetch = [&](int c) { pl.fetch(c & 1, r.start + r.warp_position(tile_of(c)), r.warp_position(tile_of(c))); };
    Map total = {1.f, 0.f, 0.f};
    const float *from = UP ? p.s0 : p.ds_end;
    if (end && r.real && from) { HN_G(from + r.row, 4); total.S = from[r.row]; }
    if (tiles) fetch(0);                                     // (every one of them has copies: the c-th is its stage's c/2-th)
    for (int c = 0; c < tiles; ++c) {
        const int j = tile_of(c), t0 = r.position(j), turn = c & 1, lo = max(0, -t0), hi = min(E, r.len - t0);
        const long long i = r.start + t0;
        __syncwarp();                                        // (the other stage has been read)
        if (c + 1 < tiles) fetch(c + 1);
        if (!pl.wait(turn, c >> 1 & 1, r.warp_position(j), is_late(p, j))) {
            pl.drain(turn, c >> 1 & 1, r.warp_position(j));
            if (c + 1 < tiles) pl.drain(turn ^ 1, (c + 1) >> 1 & 1, r.warp_position(tile_of(c + 1)));
            break;
        }
        Map own = {1.f, 0.f, 0.f};
        if (lo < hi) {
            f2 a[N], na[N], u[N], x[N];
            pl.get(turn, 0, i, u); pl.get(turn, 1, i, x);
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = mul2(u[e], x[e]);
            pl.get(turn, 2, i, x);
            if (lo > 0 || hi < E) { mask(u, lo, hi, 0.f); mask(x, lo, hi, no_decay<DECAY>()); }
            decays<DECAY>(x, a, na, own.A, own.P);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (UP) own.S = fmaf(a[e].y, fmaf(a[e].x, own.S, u[e].x), u[e].y);
                else own.S = a[N - 1 - e].x * (u[N - 1 - e].x + a[N - 1 - e].y * (u[N - 1 - e].y + own.S));
        }
        const Map inc = scan_lanes<32, UP>(own, pl.lane);
        total = compose(total, inc);                         // (of use in the last lane on the way)
    }
    total.S += pl.none;
    if (r.real && pl.lane == (UP ? 31 : 0)) {
        float4 *f = p.maps + r.row * p.segments + r.segment;
        HN_G(f, 16);
        *f = make_float4(total.A, total.P, total.S, 0.f);
    }
    if (!pl.good()) atomicExch(&hn_rec_status, 1);
}

template <typename T, int DECAY, int OCT, int LANES, bool STAGED>
__global__ void __launch_bounds__(RowLane<LANES>::kThreads, LANES > 32 ? 768 / LANES : 6) recurrence_forward_kernel(RecArgs p)
{
    using R = RowLane<LANES>;
    constexpr int E = 8 * OCT, N = E / 2;
    using Pl = Places<T, OCT, 4, R::kThreads, STAGED>;
    extern __shared__ __align__(16) char stages[];
    __shared__ Meeting<LANES> meeting;
    __shared__ uint64_t barriers[STAGED ? 3 * R::kThreads / 32 : 1];
    const T *q = (const T *)p.q, *k = (const T *)p.k, *v = (const T *)p.v, *g = (const T *)p.g;
    T *y = (T *)p.y;
    pdl_join();
    const Row<LANES, E> r(p);
    float state = 0.f;
    if (r.real && p.s0 && p.segments == 1) { HN_G(p.s0 + r.row, 4); state = p.s0[r.row]; }
    if (STAGED && LANES > 32 && threadIdx.x == 0) meeting.carry[1] = state;      // (read behind the first tile's barrier)
    Pl pl;
    pl.in[0] = k; pl.in[1] = v; pl.in[2] = g; pl.in[3] = q;
    pl.init(stages, barriers, r.len, p.n);
    auto first = [&](int j) { return r.warp_position(j); };
    if (STAGED && r.first < r.last) pl.fetch(0, r.start + first(r.first), first(r.first));
    if (LANES == 32 && p.segments > 1) state = r.template entering<true>(p);
    for (int j = r.first; j < r.last; ++j) {
        const int th = j * LANES + r.l, t0 = th * E - r.lead, met = j - r.first, turn = met & 1;
        const long long i = r.start + t0;
        const int lo = max(0, -t0), hi = min(E, r.len - t0);
        if (STAGED) {
            pl.stage_free();
            if (j + 1 < r.last && pl.good()) pl.fetch(turn ^ 1, r.start + first(j + 1), first(j + 1));
            if (!pl.wait(turn, met >> 1 & 1, first(j), is_late(p, j))) pl.keep_late(j);
        }
        const bool some = lo < hi, whole = lo == 0 && hi == E;
        f2 out[N];
        if (LANES <= 32 || j < r.live) {
            f2 a[N], u[N];
            Map own = {1.f, 0.f, pl.none};
            if (some) {
                f2 x[N], na[N];
                pl.get(turn, 0, i, u); pl.get(turn, 1, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) u[e] = mul2(u[e], x[e]);
                pl.get(turn, 2, i, x);
                if (!whole) { mask(u, lo, hi, 0.f); mask(x, lo, hi, no_decay<DECAY>()); }
                decays<DECAY>(x, a, na, own.A, own.P);
#pragma unroll
                for (int e = 0; e < N; ++e) own.S = fmaf(a[e].y, fmaf(a[e].x, own.S, u[e].x), u[e].y);
            }
            const Step<LANES, true> step(own);
            if constexpr (LANES > 32) {
                step.leave(meeting, met);
                __syncthreads();
                if (STAGED || met) state = meeting.carry[(met - 1) & 1];
            }
            float s = step.enter(meeting, met, state);
            if (p.marks && r.real && th * OCT % kMarkOctets == 0 && th * OCT / kMarkOctets < p.marks_row) {
                float *m = p.marks + r.row * p.marks_row + th * OCT / kMarkOctets;
                HN_G(m, 4);
                *m = s;
            }
            if (some) {
                pl.get(turn, 3, i, out);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float first = fmaf(a[e].x, s, u[e].x);
                    s = fmaf(a[e].y, first, u[e].y);
                    out[e] = mul2(out[e], make2(first, s));
                }
                if (!whole) mask(out, lo, hi, 0.f);
            }
            if (LANES > 32 && threadIdx.x == LANES - 1) meeting.carry[turn] = state = s;
        }
        if (!some) mask(out, 0, 0, 0.f);
        if (r.real && pl.good()) pl.put(turn, 0, y, r.start + first(j), first(j), i, t0, p.L, out);
        pl.put_done();
    }
    if (STAGED && LANES > 32 && r.first >= r.live) { __syncthreads(); state = meeting.carry[1]; }       // (no tile has a position)
    if (r.real && p.s_end && r.segment == p.segments - 1 && r.l == (LANES > 32 ? LANES - 1 : 0)) { HN_G(p.s_end + r.row, 4); p.s_end[r.row] = state; }
    if (STAGED && pl.lane == 0) tma_wait_all0();
    if (!pl.good()) {
        const int j = pl.late(), met = j - r.first;
        pl.drain(met & 1, met >> 1 & 1, first(j));
        if (j + 1 < r.last) pl.drain((met + 1) & 1, (met + 1) >> 1 & 1, first(j + 1));
        atomicExch(&hn_rec_status, 1);
    }
}

template <typename T, int DECAY, int OCT, int LANES, bool STAGED>
__global__ void __launch_bounds__(RowLane<LANES>::kThreads, LANES > 32 ? 512 / LANES : 4) recurrence_backward_kernel(RecArgs p)
{
    using R = RowLane<LANES>;
    constexpr int E = 8 * OCT, N = E / 2;
    using Pl = Places<T, OCT, 5, R::kThreads, STAGED>;
    extern __shared__ __align__(16) char stages[];
    __shared__ Meeting<LANES> along;                         // the states, from each tile's mark
    __shared__ uint64_t barriers[STAGED ? 3 * R::kThreads / 32 : 1];
    __shared__ Meeting<LANES> back;                          // the gradients of the states, from the row's end
    const T *q = (const T *)p.q, *k = (const T *)p.k, *v = (const T *)p.v, *g = (const T *)p.g, *dy = (const T *)p.dy;
    pdl_join();
    const Row<LANES, E> r(p);
    float mu = 0.f;                                          // a_{t+1} lam_{t+1} of the position behind the tile
    if (r.real && p.ds_end && p.segments == 1) { HN_G(p.ds_end + r.row, 4); mu = p.ds_end[r.row]; }
    if (STAGED && LANES > 32 && threadIdx.x == 0) back.carry[1] = mu;
    auto mark_of = [&](int j) {                              // in front of a tile
        const int mark = STAGED ? j * LANES * OCT / kMarkOctets : 0;
        if (j < 0 || !r.real || mark >= p.marks_row) return 0.f;
        const float *m = p.marks + r.row * p.marks_row + mark;
        HN_G(m, 4);
        return __ldg(m);
    };
    Pl pl;
    pl.in[0] = k; pl.in[1] = v; pl.in[2] = g; pl.in[3] = q; pl.in[4] = dy;
    pl.init(stages, barriers, r.len, p.n);
    auto first = [&](int j) { return r.warp_position(j); };
    float mark = mark_of(r.last - 1);
    // the last tile that this warp has copies of: the phases of the stages count from there
    const int top = min(r.last, (r.len + r.lead - (r.l - pl.lane) * E + Row<LANES, E>::kTile - 1) / Row<LANES, E>::kTile) - 1;
    if (STAGED && r.first < r.last) pl.fetch((r.last - 1) & 1, r.start + first(r.last - 1), first(r.last - 1));
    if (LANES == 32 && p.segments > 1) mu = r.template entering<false>(p);
    for (int j = r.last - 1; j >= r.first; --j) {
        const int t0 = r.position(j);
        const long long i = r.start + t0;
        const int lo = max(0, -t0), hi = min(E, r.len - t0);
        float from = mark;
        if (STAGED) {
            pl.stage_free();
            if (j > r.first && pl.good()) pl.fetch((j - 1) & 1, r.start + first(j - 1), first(j - 1));
            mark = mark_of(j - 1);
            if (!pl.wait(j & 1, (top - j) >> 1 & 1, first(j), is_late(p, j))) {
                pl.drain(j & 1, (top - j) >> 1 & 1, first(j));
                if (j > r.first) pl.drain((j - 1) & 1, (top - j + 1) >> 1 & 1, first(j - 1));
            }
        }
        const bool some = lo < hi, whole = lo == 0 && hi == E;
        if (LANES <= 32 || j < r.live) {
            const int met = min(r.live, r.last) - 1 - j;
            f2 a[N], na[N], w[N], u[N];
            Map own = {1.f, 0.f, pl.none}, rev = {1.f, 0.f, pl.none};
            if (some) {
                f2 x[N];
                pl.get(j & 1, 0, i, u); pl.get(j & 1, 1, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) u[e] = mul2(u[e], x[e]);
                pl.get(j & 1, 3, i, w); pl.get(j & 1, 4, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) w[e] = mul2(w[e], x[e]);
                pl.get(j & 1, 2, i, x);
                if (!whole) { mask(u, lo, hi, 0.f); mask(w, lo, hi, 0.f); mask(x, lo, hi, no_decay<DECAY>()); }
                decays<DECAY>(x, a, na, own.A, own.P);
                rev.A = own.A; rev.P = own.P;
#pragma unroll
                for (int e = 0; e < N; ++e) own.S = fmaf(a[e].y, fmaf(a[e].x, own.S, u[e].x), u[e].y);
#pragma unroll
                for (int e = N - 1; e >= 0; --e) rev.S = a[e].x * (w[e].x + a[e].y * (w[e].y + rev.S));
            }
            const Step<LANES, true> ahead(own);
            const Step<LANES, false> behind(rev);
            if constexpr (LANES > 32) {
                ahead.leave(along, met);
                behind.leave(back, met);
                __syncthreads();
                if (STAGED || met) mu = back.carry[(met - 1) & 1];
            }
            float s = ahead.enter(along, met, from);
            float m = behind.enter(back, met, mu);
            auto put = [&](T *to, int place, f2 (&f)[N]) {
                if (!whole) mask(f, lo, hi, 0.f);
                if (r.real && pl.good()) pl.put(j & 1, place, to, r.start + first(j), first(j), i, t0, p.L, f);
            };
            // (lanes without a position take part in the stores and write zeros)
            f2 x[N];
            if (some) {
                pl.get(j & 1, 4, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float mid = fmaf(a[e].x, s, u[e].x), end = fmaf(a[e].y, mid, u[e].y);
                    u[e] = make2(s, mid);                    // from here the state in front of each position
                    x[e] = mul2(x[e], make2(mid, end));
                    s = end;
                }
            }
            put((T *)p.dq, 4, x);
            if (some) {
#pragma unroll
                for (int e = N - 1; e >= 0; --e) {           // w: from here lam
                    w[e].y += m;
                    w[e].x = fmaf(a[e].y, w[e].y, w[e].x);
                    m = a[e].x * w[e].x;
                    u[e] = mul2(u[e], w[e]);
                    if (DECAY == DECAY_LOG) u[e] = mul2(u[e], a[e]);
                    if (DECAY == DECAY_SIGMOID) u[e] = mul2(u[e], mul2(a[e], na[e]));
                }
            }
            put((T *)p.dg, 2, u);
            if (some) {
                pl.get(j & 1, 1, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = mul2(x[e], w[e]);
            }
            put((T *)p.dk, 1, x);
            if (some) {
                pl.get(j & 1, 0, i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = mul2(x[e], w[e]);
            }
            put((T *)p.dv, 0, x);
            if (LANES > 32 && threadIdx.x == 0) back.carry[met & 1] = mu = m;
        } else if (r.real && pl.good()) {
            f2 zero[N];
#pragma unroll
            for (int e = 0; e < N; ++e) zero[e] = pair(0.f);
            pl.put(j & 1, 4, (T *)p.dq, r.start + first(j), first(j), i, t0, p.L, zero);
            pl.put(j & 1, 1, (T *)p.dk, r.start + first(j), first(j), i, t0, p.L, zero);
            pl.put(j & 1, 0, (T *)p.dv, r.start + first(j), first(j), i, t0, p.L, zero);
            pl.put(j & 1, 2, (T *)p.dg, r.start + first(j), first(j), i, t0, p.L, zero);
        }
        pl.put_done();
    }
    if (STAGED && LANES > 32 && r.first >= r.live) { __syncthreads(); mu = back.carry[1]; }
    if (r.real && p.ds0 && r.segment == 0 && r.l == 0) { HN_G(p.ds0 + r.row, 4); p.ds0[r.row] = mu; }
    if (STAGED && pl.lane == 0) tma_wait_all0();
    if (!pl.good()) atomicExch(&hn_rec_status, 1);
}

// a s + u for one token.  A decay next to 1 loses what it is in its own rounding (exp(-1e-6) is off by 2 % of its distance from 1, and
// 40000 tokens one by one by 5e-4 of the state): there it is s + (a - 1) s + u with a - 1 as precise as a number of its own, and the
// sum's is the one rounding of the state's size.  An infinite state stays one.  The call is a launch whatever it computes.
template <int DECAY> __device__ __forceinline__ float step_state(float g, float s, float u)
{
    if constexpr (DECAY == DECAY_VALUE) return fmaf(g, s, u);
    float a, less;                                           // a, and a - 1 where a is above a half
    bool close;
    if constexpr (DECAY == DECAY_LOG) {
        close = g > -0.6931472f;
        a = expf(g);
        less = expm1f(g);
    } else {
        const float e = expf(-fabsf(g)), x = e / (1.f + e);
        close = g >= 0.f;
        a = close ? 1.f - x : x;
        less = -x;
    }
    return close && fabsf(s) <= 3.402823466e38f ? s + fmaf(less, s, u) : fmaf(a, s, u);
}

// One token: a thread per channel.
template <typename T, int DECAY> __global__ void __launch_bounds__(256) recurrence_step_kernel(RecArgs p)
{
    pdl_join();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.rows) return;
    float s = 0.f, out = 0.f;
    if (p.s0) { HN_G(p.s0 + i, 4); s = p.s0[i]; }
    bool in = true;
    if (p.lengths) {
        const int b = (int)(i / p.C);
        HN_G(p.lengths + b, 4);
        in = __ldg(p.lengths + b) > 0;
    }
    if (in) {
        s = step_state<DECAY>(IO<T>::ld((const T *)p.g, i), s, IO<T>::ld((const T *)p.k, i) * IO<T>::ld((const T *)p.v, i));
        out = IO<T>::ld((const T *)p.q, i) * s;
    }
    IO<T>::st((T *)p.y, i, out);
    if (p.s_end) { HN_G(p.s_end + i, 4); p.s_end[i] = s; }
}

template <auto FN, int LANES, int BYTES> static int launch_rows(const RecArgs &a, cudaStream_t st)
{
    using R = RowLane<LANES>;
    const long long blocks = (a.rows + R::kRows - 1) / R::kRows * a.segments;
    if (blocks > 0x7fffffffll) return kTooLarge;
    static PerDevice ready;
    if (BYTES > 32 * 1024 && !ready.once([] { return cudaFuncSetAttribute(FN, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES) == cudaSuccess ? 1 : -1; })) return kNoLaunch;
    launch_pdl(FN, dim3((unsigned)blocks), R::kThreads, BYTES, st, a);
    return 0;
}
template <typename T, int DECAY, bool BWD, int OCT, int LANES, bool STAGED> static int launch_lanes(const RecArgs &a, cudaStream_t st)
{
    constexpr int THREADS = RowLane<LANES>::kThreads;
    if constexpr (STAGED && LANES == 32)
        if (a.segments > 1)
            if (const int e = launch_rows<recurrence_maps_kernel<T, DECAY, OCT, !BWD>, LANES, 2 * Places<T, OCT, 3, THREADS, true>::STAGE>(a, st)) return e;
    if constexpr (BWD) return launch_rows<recurrence_backward_kernel<T, DECAY, OCT, LANES, STAGED>, LANES, 2 * Places<T, OCT, 5, THREADS, STAGED>::STAGE>(a, st);
    else return launch_rows<recurrence_forward_kernel<T, DECAY, OCT, LANES, STAGED>, LANES, 2 * Places<T, OCT, 4, THREADS, STAGED>::STAGE>(a, st);
}

// Rows that leave places free are cut into segments, one warp each, as many as run at once: the second reading of two (backward: three)
// tensors costs less than the idle places, forward below 128 rows, backward below two an SM.  64 rows of 65536, bf16: 22 and 28 us,
// whole rows 34 and 82; 180 rows of 262144: 148 and 202, whole 139 and 348; 256 rows of 65536, fp32: 105 and 142, whole 68 and 166.  A row of
// fewer than 32 tiles of a warp is walked as fast by one CTA (20 rows of 5000, bf16: 8 and 12 us, in segments 13 and 15).
static int segments_of(long long rows, int L, int dtype, bool backward)
{
    const int tile = 32 * (dtype == HYENAND_F32 ? 8 : 16);
    const long long tiles = ((long long)L + (L % 8 ? 7 : 0) + tile - 1) / tile, places = (backward ? 512 : 768) / 32 * kSms;
    if (rows >= (backward ? 2 * kSms : 128) || tiles < 32) return 1;
    const long long n = places / rows, each = (tiles + n - 1) / n;
    return (int)((tiles + (each > 2 ? each : 2) - 1) / (each > 2 ? each : 2));       // (none of them empty)
}

// Lanes of a row: as few as hold it in one tile, a CTA that walks it where it is longer.
template <typename T, int DECAY, bool BWD> static int launch_recurrence_td(const RecArgs &a, cudaStream_t st)
{
    constexpr int LONG = sizeof(T) == 2 ? 2 : 1;             // octets of a thread where a row is long
    const int octets = (a.L + (a.L % 8 ? 7 : 0) + 7) / 8;    // that a row touches, wherever in one it starts
#define HN_REC(OCT, LANES, STAGED) return launch_lanes<T, DECAY, BWD, OCT, LANES, STAGED>(a, st)
    if (octets <= 4) HN_REC(1, 4, false);
    if (octets <= 8) HN_REC(1, 8, false);
    if (octets <= 16) HN_REC(1, 16, false);
    if (octets <= 32) HN_REC(1, 32, false);
    if (octets <= 64) HN_REC(1, 64, false);
    if (a.segments > 1) HN_REC(LONG, 32, true);
    if constexpr (LONG == 2) if (octets <= 128) HN_REC(2, 64, true);
    const int threads = (octets + LONG - 1) / LONG;
    // Rows that fill the GPU: one CTA each, of as many lanes as still lets all of them run at once (768 threads an SM forward, 512
    // backward), and small ones where they come in several waves anyhow.  512 rows of 65536, bf16, forward: 128 lanes 73 us, 192 70,
    // 256 (a second wave of 68) 86; backward 119, 145, 129.  12288 rows of 2000, bf16: 32 lanes 49 and 88 us, 64 52 and 100, 128 (one
    // tile, nothing travels ahead) 62 and 117; of 1531, fp32, 128 lanes 76 and 148 (32, which fp32 rows above 1024 do not take, 72 and
    // 127).  8192 rows of 8192, bf16: 32 lanes 121 and 213, 64 117 and 201, 128 117 and 215.
    // At the borders, rows of 65536, bf16 (in brackets what the rule does not take): forward 444 rows by 256 lanes 60 us (128: 66), 450 by
    // 192 69 (128: 72, 256: 77), 592 by 192 78 (128: 74), 600 by 128 83 (256: 86), 1000 by 128 155 (256: 127), 1800 by 64 262 (256: 201, 32:
    // 211): long rows of more than some 800 leave time there.  Backward 592 by 128 122 (256: 131), 600 by 256 171 (128: 188), 888 by 256 192
    // (128: 212), 1184 by 64 252 (128: 240).  fp32, rows of 32768, backward: 600 by 256 170 (128: 131), 888 by 256 181 (128: 248).
    constexpr int PLACES = BWD ? 512 : 768;
    if (threads <= 128 && a.rows >= PLACES / 64 * kSms) HN_REC(LONG, 32, true);
    if constexpr (LONG == 2) {
        if (a.rows >= PLACES / 64 * kSms) HN_REC(LONG, 64, true);
        if constexpr (!BWD) if (threads > 128 && a.rows > 3 * kSms && a.rows <= 4 * kSms) HN_REC(LONG, 192, true);
    }
    const bool two = BWD ? a.rows > 4 * kSms && a.rows <= 8 * kSms : a.rows <= 3 * kSms;
    if (threads <= 128 || !two) HN_REC(LONG, 128, true);
    HN_REC(LONG, 256, true);
#undef HN_REC
}

template <bool BWD> static int launch_recurrence(const RecArgs &a, int decay, int dtype, cudaStream_t st)
{
    if (dtype == HYENAND_F32)
        return decay == DECAY_VALUE ? launch_recurrence_td<float, DECAY_VALUE, BWD>(a, st)
               : decay == DECAY_LOG ? launch_recurrence_td<float, DECAY_LOG, BWD>(a, st) : launch_recurrence_td<float, DECAY_SIGMOID, BWD>(a, st);
    return decay == DECAY_VALUE ? launch_recurrence_td<bf16, DECAY_VALUE, BWD>(a, st)
           : decay == DECAY_LOG ? launch_recurrence_td<bf16, DECAY_LOG, BWD>(a, st) : launch_recurrence_td<bf16, DECAY_SIGMOID, BWD>(a, st);
}

static int launch_step(const RecArgs &a, int decay, int dtype, cudaStream_t st)
{
    const long long blocks = (a.rows + 255) / 256;
    if (blocks > 0x7fffffffll) return kTooLarge;
    void (*fn)(RecArgs) = dtype == HYENAND_F32
        ? (decay == DECAY_VALUE ? recurrence_step_kernel<float, DECAY_VALUE> : decay == DECAY_LOG ? recurrence_step_kernel<float, DECAY_LOG> : recurrence_step_kernel<float, DECAY_SIGMOID>)
        : (decay == DECAY_VALUE ? recurrence_step_kernel<bf16, DECAY_VALUE> : decay == DECAY_LOG ? recurrence_step_kernel<bf16, DECAY_LOG> : recurrence_step_kernel<bf16, DECAY_SIGMOID>);
    launch_pdl(fn, dim3((unsigned)blocks), 256, 0, st, a);
    return 0;
}

static int check_shape(int B, int C, int L, int decay, int dtype)
{
    if (B < 1 || C < 1 || L < 1) return fail(HYENAND_ERR_INVALID_ARG, "B, C and L must be >= 1");
    if (decay < DECAY_VALUE || decay > DECAY_SIGMOID) return fail(HYENAND_ERR_INVALID_ARG, "unknown decay %d", decay);
    if (dtype != HYENAND_F32 && dtype != HYENAND_BF16) return fail(HYENAND_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (L > (1 << 30)) return fail(HYENAND_ERR_UNSUPPORTED, "L = %d is above 2^30", L);
    if ((long long)B * C > (1ll << 28)) return fail(HYENAND_ERR_UNSUPPORTED, "B * C is above 2^28");
    return HYENAND_OK;
}

#ifdef HYENAND_DEBUG
static std::atomic<int> late_tile{-1}, late_warp{-1};
#endif
static RecArgs rec_args()
{
    RecArgs a{};
#ifdef HYENAND_DEBUG
    a.late_tile = late_tile; a.late_warp = late_warp;
#endif
    return a;
}

// marks of a row: one in front of every tile of kMarkOctets octets a row of L positions can touch
static int marks_of(int L) { return (int)(((long long)L + 7 + 8 * kMarkOctets - 1) / (8 * kMarkOctets)); }

}  // namespace hn

using namespace hn;

extern "C" long long hyenand_recurrence_marks(int L) { return L < 1 || L > (1 << 30) ? 0 : marks_of(L); }

extern "C" long long hyenand_recurrence_workspace_bytes(int B, int C, int L, int dtype)
{
    if (B < 1 || C < 1 || L < 1 || L > (1 << 30)) return 0;
    const long long rows = (long long)B * C, f = segments_of(rows, L, dtype, false), b = segments_of(rows, L, dtype, true), most = f > b ? f : b;
    return most > 1 ? rows * most * (long long)sizeof(float4) : 0;
}

extern "C" int hyenand_debug_recurrence_late(int tile, int warp)
{
#ifdef HYENAND_DEBUG
    late_tile = tile; late_warp = warp;
    return 0;
#else
    (void)tile; (void)warp;
    return -1;
#endif
}

extern "C" int hyenand_recurrence_device_status(void)
{
    int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, hn_rec_status, sizeof(int)) != cudaSuccess) return -1;
    return v;
}

extern "C" int hyenand_recurrence_forward(int B, int C, int L, int decay, int dtype, const void *q, const void *k, const void *v,
                                          const void *g, const float *s0, const int *lengths, void *y, float *s_end, float *marks,
                                          void *workspace, void *cuda_stream)
{
    clear_error();
    if (int e = check_shape(B, C, L, decay, dtype)) return e;
    if (!q || !k || !v || !g || !y) return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, g, y must be non-NULL");
    RecArgs a = rec_args();
    a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = s0; a.lengths = lengths; a.y = y; a.s_end = s_end; a.marks = marks;
    a.rows = (long long)B * C; a.n = a.rows * L; a.C = C; a.L = L; a.marks_row = marks_of(L);
    a.segments = segments_of(a.rows, L, dtype, false); a.maps = (float4 *)workspace;
    if (a.segments > 1 && !workspace) return fail(HYENAND_ERR_INVALID_ARG, "workspace must be non-NULL for this shape");
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb);
    c.in("s0", s0, rb, 4); c.in("lengths", lengths, (size_t)B * sizeof(int), 4);
    c.out("y", y, nb); c.out("s_end", s_end, rb, 4, "s0 q k v g"); c.out("marks", marks, rb * a.marks_row, 4);
    if (a.segments > 1) c.out("workspace", workspace, (size_t)a.rows * a.segments * sizeof(float4));
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_recurrence<false>(a, decay, dtype, (cudaStream_t)cuda_stream));
}

extern "C" int hyenand_recurrence_backward(int B, int C, int L, int decay, int dtype, const void *q, const void *k, const void *v,
                                           const void *g, const int *lengths, const float *marks, const void *dy, const float *ds_end,
                                           void *dq, void *dk, void *dv, void *dg, float *ds0, void *workspace, void *cuda_stream)
{
    clear_error();
    if (int e = check_shape(B, C, L, decay, dtype)) return e;
    if (!q || !k || !v || !g || !marks || !dy || !dq || !dk || !dv || !dg)
        return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, g, marks, dy, dq, dk, dv, dg must be non-NULL");
    RecArgs a = rec_args();
    a.q = q; a.k = k; a.v = v; a.g = g; a.lengths = lengths; a.marks = (float *)marks; a.dy = dy; a.ds_end = ds_end;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.ds0 = ds0;
    a.rows = (long long)B * C; a.n = a.rows * L; a.C = C; a.L = L; a.marks_row = marks_of(L);
    a.segments = segments_of(a.rows, L, dtype, true); a.maps = (float4 *)workspace;
    if (a.segments > 1 && !workspace) return fail(HYENAND_ERR_INVALID_ARG, "workspace must be non-NULL for this shape");
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb); c.in("dy", dy, nb);
    c.in("lengths", lengths, (size_t)B * sizeof(int), 4); c.in("marks", marks, rb * a.marks_row, 4); c.in("ds_end", ds_end, rb, 4);
    c.out("dq", dq, nb); c.out("dk", dk, nb); c.out("dv", dv, nb); c.out("dg", dg, nb); c.out("ds0", ds0, rb, 4, "ds_end q k v g dy marks");
    if (a.segments > 1) c.out("workspace", workspace, (size_t)a.rows * a.segments * sizeof(float4));
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_recurrence<true>(a, decay, dtype, (cudaStream_t)cuda_stream));
}

extern "C" int hyenand_recurrence_step(int B, int C, int decay, int dtype, const void *q, const void *k, const void *v, const void *g,
                                       const float *state, const int *active, void *y, float *new_state, void *cuda_stream)
{
    clear_error();
    if (int e = check_shape(B, C, 1, decay, dtype)) return e;
    if (!q || !k || !v || !g || !state || !y || !new_state)
        return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, g, state, y, new_state must be non-NULL");
    RecArgs a = rec_args();
    a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = state; a.lengths = active; a.y = y; a.s_end = new_state;
    a.rows = a.n = (long long)B * C; a.C = C; a.L = 1; a.segments = 1;
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb);
    c.in("state", state, rb, 4); c.in("active", active, (size_t)B * sizeof(int), 4);
    c.out("y", y, nb); c.out("new_state", new_state, rb, 4, "state q k v g");          // (an element a thread)
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_step(a, decay, dtype, (cudaStream_t)cuda_stream));
}
