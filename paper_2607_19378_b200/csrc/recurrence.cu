// The gated linear recurrence along the last axis, forward, backward and for one token:
//
//     s_t = a_t s_{t-1} + k_t v_t,      y_t = q_t s_t,      a_t = g_t | exp(g_t) | sigmoid(g_t)
//
// One pass over the data.  Maps s -> A s + S of neighbouring positions compose to (A1 A2, S2 + A2 S1); a thread composes the eight of
// its octet, the lanes of a row scan those by shuffles, the warps of a row meet in shared memory, and then every thread runs its
// eight steps from the state that enters them.  Long rows are walked tile by tile, the state carried in a register.  Where there are
// fewer rows than the SMs can hold, a cluster of CTAs shares a row's tiles and the maps travel through distributed shared memory.
//
// All states and maps are fp32.  A product of thousands of decays close to 1 would collect the rounding of each of them, always to
// the same side where the decay is constant; the maps therefore carry P = A - 1 beside A (P1 P2 + P1 + P2), built from 1 - a_t
// (sigmoid), from the sum of the g_t (exp), and use whichever of the two is the precise one.
#include <cooperative_groups.h>

#include "entry.cuh"
#include "octet.cuh"

namespace cg = cooperative_groups;

namespace hn {

constexpr int kMarkOctets = 128;          // the state is marked in front of every 1024 positions of a row (octets of the flat tensor)

enum { DECAY_VALUE = 0, DECAY_LOG = 1, DECAY_SIGMOID = 2 };

struct RecArgs {
    const void *q, *k, *v, *g, *dy;
    const float *s0, *ds_end;             // [rows] or nullptr: zero
    const int *lengths;                   // [B] or nullptr: L
    void *y, *dq, *dk, *dv, *dg;
    float *s_end, *ds0;                   // [rows] or nullptr
    float *marks;                         // [rows][marks_row] or nullptr (forward); read by the backward
    long long rows, n;                    // n = rows * L
    int C, L, marks_row;
};

struct Map { float A, P, S; };            // s -> (1 + P) s + S, A = 1 + P
__device__ __forceinline__ float apply(const Map &m, float s)
{
    const bool small = m.A < 0.5f;
    return fmaf(small ? m.A : m.P, s, small ? 0.f : s) + m.S;
}
// a first, then b
__device__ __forceinline__ Map compose(const Map &a, const Map &b) { return {a.A * b.A, fmaf(a.P, b.P, a.P + b.P), apply(b, a.S)}; }

// a_t and 1 - a_t (LOG: not needed, 0)
template <int DECAY, bool FAST> __device__ __forceinline__ void decay(float g, float &a, float &na)
{
    if constexpr (DECAY == DECAY_VALUE) { a = g; na = 1.f - g; }
    else if constexpr (DECAY == DECAY_LOG) { a = FAST ? __expf(g) : expf(g); na = 0.f; }
    else {
        const float e = FAST ? __expf(-fabsf(g)) : expf(-fabsf(g)), r = FAST ? __fdividef(1.f, 1.f + e) : __frcp_rn(1.f + e), x = e * r;
        a = g >= 0.f ? r : x;
        na = g >= 0.f ? x : r;
    }
}

// A row's live octet, positions [t0, t0 + 8): a, 1 - a, u for its live elements [lo, hi), the identity elsewhere; and A, P of the whole.
template <int DECAY, bool FAST>
__device__ __forceinline__ void decays(const float (&g)[8], int lo, int hi, float (&a)[8], float (&na)[8], float &A, float &P)
{
    A = 1.f; P = 0.f;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool in = e >= lo && e < hi;
        decay<DECAY, FAST>(g[e], a[e], na[e]);
        if (!in) { a[e] = 1.f; na[e] = 0.f; }
        A *= a[e];
        if constexpr (DECAY == DECAY_LOG) sum += in ? g[e] : 0.f;
        else P = fmaf(P, a[e], -na[e]);
    }
    if constexpr (DECAY == DECAY_LOG) P = expm1f(sum);
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

// Where a thread stands: LANES lanes share a row (a part of a warp, or a CTA of LANES threads), CL CTAs in a row of tiles.
template <int LANES, int CL> struct RowLane {
    static constexpr int kThreads = LANES <= 32 ? 128 : LANES;
    static constexpr int kRows = LANES <= 32 ? kThreads / LANES : 1;
    static constexpr int kWarpLanes = LANES < 32 ? LANES : 32;
    static constexpr int kWarps = LANES <= 32 ? 1 : LANES / 32;      // of one CTA, that share a row
    static constexpr int kSpan = LANES * CL;                         // octets of a tile
};

// From the maps of this thread's octets and the state that enters the tile: the state that enters the thread's octet, and `carry`
// moved on to the one that leaves the tile.  Warps meet in slots[parity], which the caller alternates.
template <int LANES, int CL, bool UP>
__device__ __forceinline__ float enter(const Map &own, float &carry, Map (*slots)[RowLane<LANES, CL>::kWarps * CL])
{
    using R = RowLane<LANES, CL>;
    const int lane = threadIdx.x % R::kWarpLanes, warp = threadIdx.x / 32;
    const Map inc = scan_lanes<R::kWarpLanes, UP>(own, lane);
    const Map before = neighbour<R::kWarpLanes, UP>(inc, lane);
    constexpr int last = UP ? R::kWarpLanes - 1 : 0;
    if constexpr (LANES <= 32) {
        const Map all = {__shfl_sync(~0u, inc.A, last, LANES), __shfl_sync(~0u, inc.P, last, LANES), __shfl_sync(~0u, inc.S, last, LANES)};
        const float s = apply(before, carry);
        carry = apply(all, carry);
        return s;
    } else {
        constexpr int N = R::kWarps * CL;
        int me = warp;
        if constexpr (CL == 1) {
            if (lane == last) slots[0][warp] = inc;
            __syncthreads();
        } else {
            auto cluster = cg::this_cluster();
            me += cluster.block_rank() * R::kWarps;
            const Map all = {__shfl_sync(~0u, inc.A, last), __shfl_sync(~0u, inc.P, last), __shfl_sync(~0u, inc.S, last)};
            if (lane < CL) cluster.map_shared_rank(&slots[0][0], lane)[me] = all;
            cluster.sync();
        }
        float in = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int j = UP ? i : N - 1 - i;
            if (j == me) in = carry;
            carry = apply(slots[0][j], carry);
        }
        return apply(before, in);
    }
}

template <typename T, int DECAY, int LANES, int CL>
__global__ void __launch_bounds__(RowLane<LANES, CL>::kThreads) recurrence_forward_kernel(RecArgs p)
{
    using R = RowLane<LANES, CL>;
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ Map slots[2][R::kWarps * CL];
    const T *q = (const T *)p.q, *k = (const T *)p.k, *v = (const T *)p.v, *g = (const T *)p.g;
    T *y = (T *)p.y;
    pdl_join();
    int rank = 0;
    if constexpr (CL > 1) {
        rank = cg::this_cluster().block_rank();
        cg::this_cluster().sync();                           // every CTA's slots exist before one is written
    }
    const long long row = (long long)(blockIdx.x / CL) * R::kRows + threadIdx.x / LANES;
    const bool real = row < p.rows;
    const int l = threadIdx.x % LANES + rank * LANES;
    int len = real ? p.L : 0;
    if (real && p.lengths) {
        const int b = (int)(row / p.C);
        HN_G(p.lengths + b, 4);
        len = max(0, min(p.L, __ldg(p.lengths + b)));
    }
    const long long start = real ? row * p.L : 0;
    const int lead = (int)(start & 7);
    float state = 0.f;
    if (real && p.s0) { HN_G(p.s0 + row, 4); state = p.s0[row]; }
    const int tiles = (lead + p.L + 8 * R::kSpan - 1) / (8 * R::kSpan);
    const int live = len ? (lead + len + 8 * R::kSpan - 1) / (8 * R::kSpan) : 0;
    for (int j = 0; j < tiles; ++j) {
        const int oct = j * R::kSpan + l, t0 = oct * 8 - lead;
        const long long i = start + t0;
        const int lo = max(0, -t0), hi = min(8, len - t0), end = min(8, p.L - t0);
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = 0.f;
        if (LANES <= 32 || j < live) {
            Octet<T> rq, rk, rv, rg;
            float a[8], na[8], u[8];
            Map own = {1.f, 0.f, 0.f};
            const bool some = lo < hi;
            if (some) {
                rk.ld(k, i, p.n); rv.ld(v, i, p.n); rg.ld(g, i, p.n); rq.ld(q, i, p.n);
                float x[8];
                rk.get(u); rv.get(x);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = e >= lo && e < hi ? u[e] * x[e] : 0.f;
                rg.get(x);
                decays<DECAY, FAST>(x, lo, hi, a, na, own.A, own.P);
#pragma unroll
                for (int e = 0; e < 8; ++e) own.S = fmaf(a[e], own.S, u[e]);
            }
            float s = enter<LANES, CL, true>(own, state, slots + (j & 1));
            if (p.marks && real && oct % kMarkOctets == 0 && oct / kMarkOctets < p.marks_row) {
                float *m = p.marks + row * p.marks_row + oct / kMarkOctets;
                HN_G(m, 4);
                *m = s;
            }
            if (some) {
                float x[8];
                rq.get(x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s = fmaf(a[e], s, u[e]);
                    out[e] = e >= lo && e < hi ? x[e] * s : 0.f;
                }
            }
        }
        if (real && lo < end) st_octet(y, i, lo, end, out);
    }
    if (real && p.s_end && l == 0) { HN_G(p.s_end + row, 4); p.s_end[row] = state; }
}

template <typename T, int DECAY, int LANES, int CL>
__global__ void __launch_bounds__(RowLane<LANES, CL>::kThreads) recurrence_backward_kernel(RecArgs p)
{
    using R = RowLane<LANES, CL>;
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ Map up[2][R::kWarps * CL], down[2][R::kWarps * CL];
    const T *q = (const T *)p.q, *k = (const T *)p.k, *v = (const T *)p.v, *g = (const T *)p.g, *dy = (const T *)p.dy;
    pdl_join();
    int rank = 0;
    if constexpr (CL > 1) {
        rank = cg::this_cluster().block_rank();
        cg::this_cluster().sync();
    }
    const long long row = (long long)(blockIdx.x / CL) * R::kRows + threadIdx.x / LANES;
    const bool real = row < p.rows;
    const int l = threadIdx.x % LANES + rank * LANES;
    int len = real ? p.L : 0;
    if (real && p.lengths) {
        const int b = (int)(row / p.C);
        HN_G(p.lengths + b, 4);
        len = max(0, min(p.L, __ldg(p.lengths + b)));
    }
    const long long start = real ? row * p.L : 0;
    const int lead = (int)(start & 7);
    float mu = 0.f;                                          // a_{t+1} lam_{t+1} of the position behind the tile
    if (real && p.ds_end) { HN_G(p.ds_end + row, 4); mu = __ldg(p.ds_end + row); }
    const int tiles = (lead + p.L + 8 * R::kSpan - 1) / (8 * R::kSpan);
    const int live = len ? (lead + len + 8 * R::kSpan - 1) / (8 * R::kSpan) : 0;
    for (int j = tiles - 1; j >= 0; --j) {
        const int oct = j * R::kSpan + l, t0 = oct * 8 - lead;
        const long long i = start + t0;
        const int lo = max(0, -t0), hi = min(8, len - t0), end = min(8, p.L - t0);
        float oq[8], ok[8], ov[8], og[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) oq[e] = ok[e] = ov[e] = og[e] = 0.f;
        if (LANES <= 32 || j < live) {
            float a[8], na[8], w[8], xk[8], xv[8], xd[8];
            Map own = {1.f, 0.f, 0.f}, back = {1.f, 0.f, 0.f};
            const bool some = lo < hi;
            float s = 0.f;
            if (real && p.marks && oct / kMarkOctets < p.marks_row) {           // (every thread of a CTA reads its tile's mark)
                const float *m = p.marks + row * p.marks_row + oct / kMarkOctets;
                HN_G(m, 4);
                s = __ldg(m);
            }
            if (some) {
                Octet<T> rq, rk, rv, rg, rd;
                rk.ld(k, i, p.n); rv.ld(v, i, p.n); rg.ld(g, i, p.n); rq.ld(q, i, p.n); rd.ld(dy, i, p.n);
                float x[8];
                rg.get(x);
                decays<DECAY, FAST>(x, lo, hi, a, na, own.A, own.P);
                back.A = own.A; back.P = own.P;
                rk.get(xk); rv.get(xv); rq.get(w); rd.get(xd);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < lo || e >= hi) xk[e] = xv[e] = w[e] = xd[e] = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) own.S = fmaf(a[e], own.S, xk[e] * xv[e]);
#pragma unroll
                for (int e = 7; e >= 0; --e) { w[e] *= xd[e]; back.S = a[e] * (w[e] + back.S); }
            }
            // the states from this CTA's mark, the gradients from the tile behind
            float in = s;
            s = enter<LANES, 1, true>(own, in, (Map(*)[RowLane<LANES, 1>::kWarps]) up[j & 1]);
            float m = enter<LANES, CL, false>(back, mu, down + (j & 1));
            if (some) {
                float before[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    before[e] = s;
                    s = fmaf(a[e], s, xk[e] * xv[e]);
                    oq[e] = xd[e] * s;
                }
#pragma unroll
                for (int e = 7; e >= 0; --e) {
                    const float lam = w[e] + m;
                    m = a[e] * lam;
                    ok[e] = lam * xv[e];
                    ov[e] = lam * xk[e];
                    const float da = lam * before[e];
                    og[e] = DECAY == DECAY_VALUE ? da : DECAY == DECAY_LOG ? da * a[e] : da * (a[e] * na[e]);
                    if (e < lo || e >= hi) og[e] = 0.f;
                }
            }
        }
        if (real && lo < end) {
            st_octet((T *)p.dq, i, lo, end, oq);
            st_octet((T *)p.dk, i, lo, end, ok);
            st_octet((T *)p.dv, i, lo, end, ov);
            st_octet((T *)p.dg, i, lo, end, og);
        }
    }
    if (real && p.ds0 && l == 0) { HN_G(p.ds0 + row, 4); p.ds0[row] = mu; }
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
        float a, na;
        decay<DECAY, false>(IO<T>::ld((const T *)p.g, i), a, na);
        s = fmaf(a, s, IO<T>::ld((const T *)p.k, i) * IO<T>::ld((const T *)p.v, i));
        out = IO<T>::ld((const T *)p.q, i) * s;
    }
    IO<T>::st((T *)p.y, i, out);
    if (p.s_end) { HN_G(p.s_end + i, 4); p.s_end[i] = s; }
}

template <int LANES, int CL> static int launch_rows(void (*fn)(RecArgs), const RecArgs &a, cudaStream_t st)
{
    using R = RowLane<LANES, CL>;
    const long long blocks = (a.rows + R::kRows - 1) / R::kRows * CL;
    if (blocks > 0x7fffffffll) return -1;
    if constexpr (CL == 1) {
        launch_pdl(fn, dim3((unsigned)blocks), R::kThreads, 0, st, a);
    } else {
        cudaLaunchConfig_t c{};
        c.gridDim = dim3((unsigned)blocks); c.blockDim = dim3(R::kThreads); c.stream = st;
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = CL; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
        c.attrs = &at; c.numAttrs = 1;
        cudaLaunchKernelEx(&c, fn, a);
    }
    return 0;
}

// Lanes of a row: as few as hold it in one tile, a CTA that walks it where it is longer.  Rows fewer than four CTAs an SM are shared
// by a cluster.
template <typename T, int DECAY, bool BWD> static int launch_recurrence_td(const RecArgs &a, cudaStream_t st)
{
    const int octets = (a.L + (a.L % 8 ? 7 : 0) + 7) / 8;
#define HN_REC(LANES, CL) return launch_rows<LANES, CL>(BWD ? recurrence_backward_kernel<T, DECAY, LANES, CL> : recurrence_forward_kernel<T, DECAY, LANES, CL>, a, st)
    if (octets <= 4) HN_REC(4, 1);
    if (octets <= 8) HN_REC(8, 1);
    if (octets <= 32) HN_REC(32, 1);
    if (octets <= 128 || a.rows >= 4 * kSms) HN_REC(128, 1);
    if (octets <= 256 || a.rows * 2 >= 4 * kSms) HN_REC(128, 2);
    if (octets <= 512 || a.rows * 4 >= 4 * kSms) HN_REC(128, 4);
    HN_REC(128, 8);
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
    if (blocks > 0x7fffffffll) return -1;
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

static int finish(int launched)
{
    if (launched < 0) return fail(HYENAND_ERR_UNSUPPORTED, "kernel grid too large for one launch");
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? HYENAND_OK : fail(HYENAND_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

// marks of a row: one in front of every tile of kMarkOctets octets a row of L positions can touch
static int marks_of(int L) { return (int)(((long long)L + 7 + 8 * kMarkOctets - 1) / (8 * kMarkOctets)); }

}  // namespace hn

using namespace hn;

extern "C" long long hyenand_recurrence_marks(int L) { return L < 1 || L > (1 << 30) ? 0 : marks_of(L); }

extern "C" int hyenand_recurrence_forward(int B, int C, int L, int decay, int dtype, const void *q, const void *k, const void *v,
                                          const void *g, const float *s0, const int *lengths, void *y, float *s_end, float *marks,
                                          void *cuda_stream)
{
    clear_error();
    if (int e = check_shape(B, C, L, decay, dtype)) return e;
    if (!q || !k || !v || !g || !y) return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, g, y must be non-NULL");
    RecArgs a{};
    a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = s0; a.lengths = lengths; a.y = y; a.s_end = s_end; a.marks = marks;
    a.rows = (long long)B * C; a.n = a.rows * L; a.C = C; a.L = L; a.marks_row = marks_of(L);
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb);
    c.in("s0", s0, rb, 4); c.in("lengths", lengths, (size_t)B * sizeof(int), 4);
    c.out("y", y, nb); c.out("s_end", s_end, rb, 4, s0); c.out("marks", marks, rb * a.marks_row, 4);
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_recurrence<false>(a, decay, dtype, (cudaStream_t)cuda_stream));
}

extern "C" int hyenand_recurrence_backward(int B, int C, int L, int decay, int dtype, const void *q, const void *k, const void *v,
                                           const void *g, const int *lengths, const float *marks, const void *dy, const float *ds_end,
                                           void *dq, void *dk, void *dv, void *dg, float *ds0, void *cuda_stream)
{
    clear_error();
    if (int e = check_shape(B, C, L, decay, dtype)) return e;
    if (!q || !k || !v || !g || !marks || !dy || !dq || !dk || !dv || !dg)
        return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, g, marks, dy, dq, dk, dv, dg must be non-NULL");
    RecArgs a{};
    a.q = q; a.k = k; a.v = v; a.g = g; a.lengths = lengths; a.marks = (float *)marks; a.dy = dy; a.ds_end = ds_end;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.ds0 = ds0;
    a.rows = (long long)B * C; a.n = a.rows * L; a.C = C; a.L = L; a.marks_row = marks_of(L);
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb); c.in("dy", dy, nb);
    c.in("lengths", lengths, (size_t)B * sizeof(int), 4); c.in("marks", marks, rb * a.marks_row, 4); c.in("ds_end", ds_end, rb, 4);
    c.out("dq", dq, nb); c.out("dk", dk, nb); c.out("dv", dv, nb); c.out("dg", dg, nb); c.out("ds0", ds0, rb, 4, ds_end);
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
    RecArgs a{};
    a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = state; a.lengths = active; a.y = y; a.s_end = new_state;
    a.rows = a.n = (long long)B * C; a.C = C; a.L = 1;
    CallTensors c;
    const size_t nb = (size_t)a.n * elsize(dtype), rb = (size_t)a.rows * sizeof(float);
    c.in("q", q, nb); c.in("k", k, nb); c.in("v", v, nb); c.in("g", g, nb);
    c.in("state", state, rb, 4); c.in("active", active, (size_t)B * sizeof(int), 4);
    c.out("y", y, nb); c.out("new_state", new_state, rb, 4, state);
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_step(a, decay, dtype, (cudaStream_t)cuda_stream));
}
