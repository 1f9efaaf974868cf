// Shared by the residual block's kernels (internal): arguments, the gate, vectors of tokens, sums over the channels of a tile.
#pragma once
#include <cooperative_groups.h>

#include "common.cuh"
#include "entry.cuh"
#include "octet.cuh"
#include "pair.cuh"
#include "philox.cuh"
#include "tile_walk.cuh"
#include "tma_util.cuh"

namespace hn {

enum { GATE_NONE = 0, GATE_SIGMOID = 1, GATE_SILU = 2 };

struct BlockArgs {
    const void *x, *m, *z, *dr, *dn;
    const float *g_post, *scale, *g_pre;      // [C] or nullptr
    float eps;
    int gate;
    DropArgs drop;
    void *r, *n, *dx, *dm, *dz;
    float *stats;                             // [2][B][T]: rho_m, rho_r
    float *partial;                           // [slots][3][C]: dg_post, dscale, dg_pre
    int B, C, T;
    long long tiles;                          // of all batch entries
    int tiles_b;                              // of one
};

// ---- tile kernels ---------------------------------------------------------------------------------------------------
//
// A thread works on four neighbouring tokens of N channels; LT lanes side by side make a tile of tokens, the other lanes and the warps
// of a CTA are channels, and a cluster of CTAs holds the channels that one does not.  A tile stays in shared memory between the sums
// over its channels and the results: each tensor is read once.

constexpr int kTileThreads = 256, kTileWarps = kTileThreads / 32;
constexpr int kBlockSlots = 4 * kSms;                       // of the workspace: sums over the tokens of so many CTAs or clusters
constexpr int kTileCtas = 8;                                 // of a cluster at most
// N at most, times the element's bytes: two stages of a tile for two CTAs in an SM's shared memory
constexpr int kForwardBytes = 16, kBackwardBytes = 8;


constexpr int V = 4, P = V / 2;                              // tokens of a thread, and pairs of them

// the smaller of two, NaN where either is (fminf takes the other)
__device__ __forceinline__ float min_or_nan(float x, float y) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y)); return r; }

// act(z), and with SLOPE act'(z).  exp(-z) is held below the largest float: where it would be infinite, sigmoid(z) is 0 and
// 1 - sigmoid(z) = exp(-z) sigmoid(z) must not be infinity times 0.
template <bool SILU, bool SLOPE> __device__ __forceinline__ void gate_pair(f2 z, f2 &a, f2 &da)
{
    float x, y;
    split2(mul2(z, pair(-1.4426950408889634f)), x, y);
    const f2 e = SLOPE ? make2(min_or_nan(ex2(x), 3e38f), min_or_nan(ex2(y), 3e38f)) : make2(ex2(x), ex2(y));
    split2(add2(e, pair(1.f)), x, y);
    const f2 s = make2(rcp(x), rcp(y));
    a = SILU ? mul2(z, s) : s;
    if (SLOPE) {
        const f2 t = mul2(e, s);
        da = SILU ? mul2(s, fma2(z, t, pair(1.f))) : mul2(s, t);
    }
}
// the same for a vector; the kind is one for the whole launch
template <bool SLOPE> __device__ __forceinline__ void gates(int kind, const f2 (&z)[P], f2 (&a)[P], f2 (&da)[P])
{
    if (kind == GATE_SILU) {
#pragma unroll
        for (int e = 0; e < P; ++e) gate_pair<true, SLOPE>(z[e], a[e], da[e]);
    } else {
#pragma unroll
        for (int e = 0; e < P; ++e) gate_pair<false, SLOPE>(z[e], a[e], da[e]);
    }
}

// The next tile travels into shared memory while this one is worked on.  A tile is ROWS * N rows (channels) of TT tokens of each
// tensor; the CTA's threads fetch it in 16-byte pieces on 16-byte boundaries of the tensor.  Where rows start inside a piece (!ALIGNED)
// there is one piece more a row, and the vectors are cut out of their neighbours.  A piece beyond the tensor's end, or beyond the
// batch entry's tokens, is filled with zeros.
template <typename T, int LT, int N, int TENSORS, bool ALIGNED> struct Stage {
    static constexpr int PER = 16 / (int)sizeof(T), TT = LT * V, ROWS = kTileThreads / LT, PIECES = TT / PER;
    static constexpr int ROW_BYTES = (PIECES + !ALIGNED) * 16, TENSOR_BYTES = ROWS * N * ROW_BYTES, BYTES = TENSORS * TENSOR_BYTES;
    static constexpr int EACH = (ROWS * N * PIECES + kTileThreads - 1) / kTileThreads;

    static __device__ __forceinline__ void piece(char *dst, const T *p, long long at, bool wanted, long long elements)
    {
        int bytes = wanted ? 16 : 0;
        if (!ALIGNED && wanted && at + PER > elements) bytes = (int)(elements - at) * (int)sizeof(T);      // (the tensor ends inside)
        if (bytes) HN_G(p + at, bytes);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(p + at), "r"(bytes) : "memory");
    }
    // the rows of the channels [first, first + mine) of a tile whose first token is element `start` of channel `first`, with `left`
    // tokens of the entry in front of it; f(tensor, pointer) is called for each tensor that there is
    template <typename F> static __device__ __forceinline__ void fetch(char *stage, long long start, int T_, int mine, int left, long long elements, F each_tensor)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = threadIdx.x + i * kTileThreads, r = q / PIECES, k = q % PIECES;
            if (ROWS * N * PIECES % kTileThreads && r >= ROWS * N) break;
            const long long row = start + (long long)r * T_;
            const int shift = ALIGNED ? 0 : (int)row & (PER - 1);
            const bool wanted = r < mine && k * PER - shift < left;
            each_tensor([&](int tensor, const void *p) { piece(stage + tensor * TENSOR_BYTES + r * ROW_BYTES + k * 16, (const T *)p, row - shift + k * PER, wanted, elements); });
        }
        if (!ALIGNED)
            for (int r = threadIdx.x; r < ROWS * N; r += kTileThreads) {
                const long long row = start + (long long)r * T_;
                const int shift = (int)row & (PER - 1);
                if (shift) each_tensor([&](int tensor, const void *p) {
                    piece(stage + tensor * TENSOR_BYTES + r * ROW_BYTES + PIECES * 16, (const T *)p, row - shift + TT, r < mine && TT - shift < left, elements); });
            }
    }
    // this thread's tokens of its channel j; start: as above, of that channel; count: tokens of the entry from this thread's on
    static __device__ __forceinline__ void get(const char *stage, int tensor, int j, long long start, int count, f2 (&f)[P])
    {
        const int tl = threadIdx.x % LT;
        const char *row = stage + tensor * TENSOR_BYTES + (j * ROWS + threadIdx.x / LT) * ROW_BYTES;
        if constexpr (ALIGNED) {
            if constexpr (sizeof(T) == 2) {
                const uint2 w = reinterpret_cast<const uint2 *>(row)[tl];
                f[0] = widen2(w.x); f[1] = widen2(w.y);
            } else {
                const float4 w = reinterpret_cast<const float4 *>(row)[tl];
                f[0] = make2(w.x, w.y); f[1] = make2(w.z, w.w);
            }
        } else {
            const int at = tl * V + ((int)start & (PER - 1));
            float v[V];
            if constexpr (sizeof(T) == 2) {
                const unsigned *w = reinterpret_cast<const unsigned *>(row) + (at >> 1);
                const unsigned odd = at & 1, last = odd ? w[2] : 0u;
                unpack2(__funnelshift_r(w[0], w[1], odd * 16), v[0], v[1]); unpack2(__funnelshift_r(w[1], last, odd * 16), v[2], v[3]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = reinterpret_cast<const float *>(row)[at + e];
            }
            if (count < V) {                                 // behind the entry's tokens come the next channel's
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = e < count ? v[e] : 0.f;
            }
            f[0] = make2(v[0], v[1]); f[1] = make2(v[2], v[3]);
        }
    }
};
__device__ __forceinline__ void stage_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void stage_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(LEFT) : "memory"); }

template <typename T, bool ALIGNED> __device__ __forceinline__ void st_vector(void *ptr, long long i, int count, const f2 (&f)[P])
{
    T *p = (T *)ptr + i;
    if constexpr (ALIGNED) {                                 // (called with whole vectors only)
        HN_G(p, V * sizeof(T));
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(narrow2(f[0]), narrow2(f[1]));
        else *reinterpret_cast<float4 *>(p) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    } else {
        float v[V];
        split2(f[0], v[0], v[1]); split2(f[1], v[2], v[3]);
        if (sizeof(T) == 2 && count >= V) {
            HN_G(p, V * sizeof(T));
            if (!(i & 1)) {
                reinterpret_cast<unsigned *>(p)[0] = pack2(v[0], v[1]);
                reinterpret_cast<unsigned *>(p)[1] = pack2(v[2], v[3]);
            } else {
                IO<T>::st(p, 0, v[0]);
                *reinterpret_cast<unsigned *>(p + 1) = pack2(v[1], v[2]);
                IO<T>::st(p, 3, v[3]);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < count) IO<T>::st(p, e, v[e]);
    }
}

// Which elements stay, bit e of keep[j] for token e of channel j; start: element of channel 0's first token of this thread, hop: from
// channel to channel.  Eight tokens share a counter: where octets hold the vectors of two neighbouring lanes, each of the two works
// out every other channel's and they exchange them.
template <int N> __device__ __forceinline__ void keep_bits(const DropKey &key, bool paired, long long start, long long hop, unsigned (&keep)[N])
{
    if constexpr (N % 2 == 0)
        if (paired) {
            const int odd = threadIdx.x & 1;
            uint4 w[N / 2];
            key.words((start + odd * hop) >> 3, hop >> 2, w);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const unsigned own = key.bits(w[j / 2]), other = __shfl_xor_sync(~0u, own, 1);
                keep[j] = (odd ? other : own) >> (4 * odd);
                keep[j + 1] = (odd ? own : other) >> (4 * odd);
            }
            return;
        }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const long long i = start + j * hop;
        const int shift = (int)(i & 7);
        keep[j] = key.keep(i >> 3) >> shift;
        if (shift + V > 8) keep[j] |= key.keep((i >> 3) + 1) << (8 - shift);
    }
}
__device__ __forceinline__ void drop_pair(unsigned keep, int e, f2 &f)
{
    f = make2(keep >> (2 * e) & 1 ? f.x : 0.f, keep >> (2 * e + 1) & 1 ? f.y : 0.f);
}
__device__ __forceinline__ void drop_pairs(unsigned keep, f2 (&f)[P])
{
#pragma unroll
    for (int e = 0; e < P; ++e) drop_pair(keep, e, f[e]);
}

// Sums over the channels of a tile's tokens: K sums of V tokens a thread -> K x TT totals of the cluster.
template <int LT, int K> struct alignas(16) TileSums {
    static constexpr int TT = LT * V, STEPS = LT == 8 ? 2 : 0;    // 32 / LT rows of channels in a warp
    static constexpr int CLS = LT == 8 ? kTileCtas : 1;
    float warp[kTileWarps][K][TT];
    float peers[2][CLS][K][TT];
    float total[K][TT];
    uint64_t arrived[2];                                     // of peers[parity]: bytes of all CTAs
    int failed;

    __device__ __forceinline__ void init()
    {
        if (threadIdx.x == 0) { mbar_init(&arrived[0], 1); mbar_init(&arrived[1], 1); failed = 0; fence_mbar_init(); }
    }
    // the lanes of a warp that hold the same tokens add up: halves of the vector change sides until one token is left a lane
    static __device__ __forceinline__ void across(float (&s)[V], int lane)
    {
        int n = V;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            const int bit = 16 >> st;
            const bool up = lane & bit;
            n /= 2;
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                if (i < n) {
                    const float give = up ? s[i] : s[n + i], keep = up ? s[n + i] : s[i];
                    s[i] = keep + __shfl_xor_sync(~0u, give, bit);
                }
        }
    }
    // The totals of the cluster's channels: `finish` is called by threads 0 .. TT - 1 with a token and its K totals; what it leaves in
    // total[][] is there for the CTA after its next barrier.  CTAs send each other their totals as asynchronous stores that a barrier
    // in the receiver's memory counts: a barrier of the whole cluster would also wait for the last tile's results to reach memory
    // (forward of 65536 tokens of 768 channels, three CTAs a cluster: 186 us with it).  A slot is written again two tiles later, which
    // takes a total of the tile between, which its reader sends after it has read.
    template <typename F> __device__ __forceinline__ void sum(const f2 (&pairs)[K][P], int ctas, int rank, int parity, unsigned phase, F finish)
    {
        constexpr int LEFT = V >> STEPS;
        const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, tl = lane % LT;
        int first = 0, n = V;                                // of the thread's tokens, those this lane is left with
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
            { n /= 2; if (lane & (16 >> st)) first += n; }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s[V];
#pragma unroll
            for (int e = 0; e < P; ++e) split2(pairs[k][e], s[2 * e], s[2 * e + 1]);
            across(s, lane);
#pragma unroll
            for (int i = 0; i < LEFT; ++i) warp[w][k][tl * V + first + i] = s[i];
        }
        __syncthreads();
        if (CLS > 1 && ctas > 1) {
            static_assert(CLS == 1 || K * TT / 4 <= 32, "one warp sends and waits");
            if (w != 0) return;
            if (lane == 0) mbar_expect_tx(&arrived[parity], ctas * K * TT * sizeof(float));
            __syncwarp();
            if (lane < K * TT / 4) {
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int j = 0; j < kTileWarps; ++j) {
                    const float4 v = reinterpret_cast<const float4 *>(&warp[j][0][0])[lane];
                    a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
                }
                const unsigned to = smem_u32(reinterpret_cast<float4 *>(&peers[parity][rank][0][0]) + lane), bar = smem_u32(&arrived[parity]);
                for (int r = 0; r < ctas; ++r) {
                    unsigned rto, rbar;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rto) : "r"(to), "r"(r));
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rbar) : "r"(bar), "r"(r));
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];\n"
                                 ::"r"(rto), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w), "r"(rbar) : "memory");
                }
            }
            if (!mbar_wait(&arrived[parity], phase)) failed = 1;
            __syncwarp();
        }
        for (int t = threadIdx.x; t < TT; t += kTileThreads) {
            float a[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                a[k] = 0.f;
                if (CLS > 1 && ctas > 1) for (int r = 0; r < ctas; ++r) a[k] += peers[parity][r][k][t];
                else
#pragma unroll
                    for (int j = 0; j < kTileWarps; ++j) a[k] += warp[j][k][t];
            }
            finish(t, a);
        }
    }
};

template <typename S> static int read_status(S &word)
{
    int v = 0;
    return cudaMemcpyFromSymbol(&v, word, sizeof(int)) == cudaSuccess ? v : -1;
}
int block_forward_status();
int block_backward_status();

// How the tile kernels take a shape (block.cu): lanes along the tokens, channels of a thread, CTAs of a cluster.
struct TileShape { int lt, n, ctas; };
// clusters launched (slots of the workspace that a backward has written), or below 0 (finish)
int launch_block_tile_forward(const BlockArgs &a, int dtype, const TileShape &s, cudaStream_t st);
int launch_block_tile_backward(const BlockArgs &a, int dtype, const TileShape &s, cudaStream_t st);

// As many clusters as run at once, each walking its share of the tiles: one more would run after all the others (98 clusters of three
// where 90 fit: twice the time).  Single CTAs are launched with the programmatic start; clusters plainly (the early start was not tried
// with them).
template <auto FN, int BYTES> static int launch_tiles(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    static PerDevice fit[kTileCtas + 1];                     // clusters of so many CTAs that run at once
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)s.ctas); c.blockDim = dim3(kTileThreads); c.stream = st; c.dynamicSmemBytes = BYTES;
    cudaLaunchAttribute at[1];
    if (s.ctas > 1) {
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = s.ctas; at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    } else {
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
    }
    c.attrs = at; c.numAttrs = 1;
    const int most = fit[s.ctas].get([&] {
        int n = 0, dev = 0, sms = kSms;
        if (cudaFuncSetAttribute(FN, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES) != cudaSuccess) return -1;
        if (s.ctas > 1) {
            if (cudaOccupancyMaxActiveClusters(&n, FN, &c) != cudaSuccess) return -1;
        } else {
            cudaGetDevice(&dev);
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, FN, kTileThreads, BYTES) != cudaSuccess) return -1;
            n *= sms;
        }
        return n < 1 ? -1 : n < kBlockSlots ? n : kBlockSlots;
    });
    if (most < 1) return kNoLaunch;
    const long long clusters = a.tiles < most ? a.tiles : most;
    c.gridDim = dim3((unsigned)(clusters * s.ctas));
    return cudaLaunchKernelEx(&c, FN, a, s.ctas) == cudaSuccess ? (int)clusters : kNoLaunch;
}

}  // namespace hn
