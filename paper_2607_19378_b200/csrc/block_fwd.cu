// The residual block's forward on tiles (block.cu has the formulas).
//
// One meeting of the cluster a tile: beside sum m^2 it gathers sum x^2, sum x b and sum b^2 with b = scale D act(z) g_post m, and since
// r = x + rho_m b,   sum r^2 = sum x^2 + 2 rho_m sum x b + rho_m^2 sum b^2.   Where the branch cancels most of x that difference
// loses what matters (below a quarter of the squares it comes from), and where m is above 1e17 or so the squares of b, which rho_m has
// not brought down yet, are infinite; such a tile meets once more and adds up r^2 itself.
//
// 44 instructions an element with gate and dropout, and 16 warps an SM (registers; two stages of three tensors in shared memory) keep the
// issue slots 45 % busy: the CTA's three barriers a tile and the meeting take the rest.  16 x 4096 tokens of 768 channels, bf16: 143 us
// (0.54 of the measured copy rate), without dropout 119 (0.65); 884736 tokens of 64, fp32, no gate: 178 (0.78).  Four lanes along the
// tokens, or half the channels a thread, and the sums of a tile worked on before the results of the one before it (24 warps an SM): 195 us
// at the least; tiles of half the tokens are rows of 32 bytes, and clusters of twice the CTAs are slower to meet.
#include "block.cuh"

namespace hn {

namespace cg = cooperative_groups;

static __device__ int hn_block_status;                       // 1: a bounded wait gave up
int block_forward_status() { return read_status(hn_block_status); }

template <typename T, int LT, int N, bool ALIGNED> __global__ void __launch_bounds__(kTileThreads, N <= 4 ? 3 : N * (int)sizeof(T) > kForwardBytes ? 1 : 2) block_tile_forward_kernel(BlockArgs p, int ctas)
{
    constexpr int TT = LT * V, ROWS = kTileThreads / LT;
    using Sums = TileSums<LT, 4>;
    using St = Stage<T, LT, N, 3, ALIGNED>;
    enum { X = 0, M = 1, Z = 2 };
    extern __shared__ __align__(16) char stages[];
    __shared__ Sums sums;
    pdl_join();
    int rank = 0;
    sums.init();
    if (LT == 8 && ctas > 1) {
        rank = cg::this_cluster().block_rank();
        cg::this_cluster().sync();                           // every CTA's barriers and slots exist before one is written
    }
    const bool drop = p.drop.threshold != 0;
    const DropKey key(drop ? DropKey(p.drop) : DropKey());
    const int row = threadIdx.x / LT, tl = threadIdx.x % LT, share = (p.C + ctas - 1) / ctas, c0 = rank * share + row;
    const int mine = min(share, p.C - rank * share);         // channels of this CTA
    const long long elements = (long long)p.B * p.C * p.T;
    float g[N], gn[N];                                       // scale g_post / (1 - p); g_pre
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int c = c0 + j * ROWS;
        const bool have = j * ROWS + row < mine;
        g[j] = drop ? p.drop.scale : 1.f; gn[j] = 0.f;
        if (have && p.g_post) { HN_G(p.g_post + c, 4); g[j] *= __ldg(p.g_post + c); }
        if (have && p.scale) { HN_G(p.scale + c, 4); g[j] *= __ldg(p.scale + c); }
        if (have && p.g_pre) { HN_G(p.g_pre + c, 4); gn[j] = __ldg(p.g_pre + c); }
    }
    const long long entry = (long long)p.C * p.T, first = (long long)c0 * p.T, hop = (long long)ROWS * p.T;
    auto fetch = [&](char *stage, const TileWalk &w) {
        if (w.inside(p.B)) {
            const int t0 = w.r * TT;
            St::fetch(stage, w.b * entry + (long long)rank * share * p.T + t0, p.T, mine, p.T - t0, elements, [&](auto piece) {
                piece(M, p.m);
                if (p.z) piece(Z, p.z);
                piece(X, p.x);
            });
        }
        stage_commit();
    };
    TileWalk here(blockIdx.x / ctas, gridDim.x / ctas, p.tiles_b), ahead = here;
    fetch(stages, ahead);
    int meeting = 0;                                         // counted: parity of its slots, phase of its barrier
    for (int turn = 0; here.inside(p.B); here.next(), turn ^= 1, ++meeting) {
        char *stage = stages + turn * St::BYTES;
        stage_wait<0>();
        __syncthreads();                                     // this tile is here, and the other stage has been read
        ahead.next();
        fetch(stages + (turn ^ 1) * St::BYTES, ahead);
        const unsigned b = here.b;
        const int t0 = here.r * TT, t = t0 + tl * V, count = p.T - t;
        const long long row0 = b * entry + first + t0;       // element where the row of this thread's first channel starts
        f2 br[N][P], s[4][P];
        unsigned keep[N];
        if (drop) keep_bits<N>(key, p.T % 8 == 0, row0 + tl * V, hop, keep);
#pragma unroll
        for (int e = 0; e < P; ++e) s[0][e] = s[1][e] = s[2][e] = s[3][e] = pair(0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const long long start = row0 + j * hop;
            f2 f[P];
            St::get(stage, M, j, start, count, f);
#pragma unroll
            for (int e = 0; e < P; ++e) { s[0][e] = fma2(f[e], f[e], s[0][e]); br[j][e] = mul2(f[e], pair(g[j])); }
            if (p.z) {
                St::get(stage, Z, j, start, count, f);
                f2 a[P], da[P];
                gates<false>(p.gate, f, a, da);
#pragma unroll
                for (int e = 0; e < P; ++e) br[j][e] = mul2(br[j][e], a[e]);
            }
            if (drop) drop_pairs(keep[j], br[j]);
            St::get(stage, X, j, start, count, f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                s[1][e] = fma2(f[e], f[e], s[1][e]);
                s[2][e] = fma2(f[e], br[j][e], s[2][e]);
                s[3][e] = fma2(br[j][e], br[j][e], s[3][e]);
            }
        }
        bool cancelled = false;
        const float inv = 1.f / (float)p.C;
        sums.sum(s, ctas, rank, meeting & 1, meeting >> 1 & 1, [&](int k, const float (&a)[4]) {
            const float rm = p.g_post ? rsqrtf(a[0] * inv + p.eps) : 1.f, bb = rm * (rm * a[3]), rr = fmaf(2.f * rm, a[2], a[1]) + bb;
            cancelled = p.g_pre && !(rr >= 0.25f * (a[1] + bb) && rr <= 3.402823466e38f);
            const float rn = rsqrtf(fmaxf(rr, 0.f) * inv + p.eps);
            sums.total[0][k] = rm;
            sums.total[1][k] = rn;
            if (p.stats && rank == 0 && t0 + k < p.T) {
                float *st = p.stats + (long long)b * p.T + t0 + k;
                if (p.g_post) { HN_G(st, 4); *st = rm; }
                if (p.g_pre) { HN_G(st + (long long)p.B * p.T, 4); st[(long long)p.B * p.T] = rn; }
            }
        });
        const bool again = __syncthreads_or(cancelled);      // (every CTA has the same totals: they agree)
        if (sums.failed) break;
        f2 rm[P];
#pragma unroll
        for (int e = 0; e < P; ++e) rm[e] = *reinterpret_cast<const f2 *>(&sums.total[0][tl * V + 2 * e]);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            f2 f[P];
            St::get(stage, X, j, row0 + j * hop, count, f);
#pragma unroll
            for (int e = 0; e < P; ++e) br[j][e] = fma2(rm[e], br[j][e], f[e]);
        }
        if (again) {
            ++meeting;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                s[0][e] = s[1][e] = s[2][e] = s[3][e] = pair(0.f);
#pragma unroll
                for (int j = 0; j < N; ++j) s[0][e] = fma2(br[j][e], br[j][e], s[0][e]);
            }
            sums.sum(s, ctas, rank, meeting & 1, meeting >> 1 & 1, [&](int k, const float (&a)[4]) {
                if (!cancelled) return;                      // (a token's result is its own: its neighbours in the tile do not change it)
                const float rn = rsqrtf(a[0] * inv + p.eps);
                sums.total[1][k] = rn;
                if (p.stats && rank == 0 && t0 + k < p.T) {
                    float *st = p.stats + ((long long)p.B + b) * p.T + t0 + k;
                    HN_G(st, 4);
                    *st = rn;
                }
            });
            __syncthreads();
            if (sums.failed) break;
        }
#pragma unroll
        for (int e = 0; e < P; ++e) rm[e] = *reinterpret_cast<const f2 *>(&sums.total[1][tl * V + 2 * e]);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j * ROWS + row >= mine || count <= 0) continue;
            const long long i = row0 + j * hop + tl * V;
            st_vector<T, ALIGNED>(p.r, i, count, br[j]);
            if (p.g_pre) {
#pragma unroll
                for (int e = 0; e < P; ++e) br[j][e] = mul2(br[j][e], mul2(rm[e], pair(gn[j])));
                st_vector<T, ALIGNED>(p.n, i, count, br[j]);
            }
        }
    }
    stage_wait<0>();
    if (LT == 8 && ctas > 1) {
        if (sums.failed && threadIdx.x == 0) atomicExch(&hn_block_status, 1);
        cg::this_cluster().sync();                           // no CTA leaves while another may still write to it
    }
}

template <typename T, int LT, int N, bool ALIGNED> static int go(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    return launch_tiles<block_tile_forward_kernel<T, LT, N, ALIGNED>, 2 * Stage<T, LT, N, 3, ALIGNED>::BYTES>(a, s, st);
}
template <typename T, int LT, int N> static int by_alignment(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    return a.T % (16 / sizeof(T)) == 0 ? go<T, LT, N, true>(a, s, st) : go<T, LT, N, false>(a, s, st);
}
// for shapes that come with rows on 16-byte boundaries only
template <typename T, int LT, int N> static int aligned_only(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    return a.T % (16 / sizeof(T)) == 0 ? go<T, LT, N, true>(a, s, st) : kNoLaunch;
}
// What tile_shape (block.cu) can ask for.  Ragged rows have half the channels a thread: of fp32 they come with 1, 2 or 4 (1 with them
// alone), of bf16 never with 6; fp32 never with 6 either (from 1025 channels on it is at least seven).
template <typename T> static int by_shape(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    constexpr bool F32 = sizeof(T) == 4;
    if (s.n == 2) return s.lt == 32 ? by_alignment<T, 32, 2>(a, s, st) : by_alignment<T, 8, 2>(a, s, st);
    if constexpr (F32) {
        if (s.n == 1) return s.lt == 32 ? by_alignment<T, 32, 1>(a, s, st) : go<T, 8, 1, false>(a, s, st);
        if (s.n == 4) return s.lt == 32 ? aligned_only<T, 32, 4>(a, s, st) : by_alignment<T, 8, 4>(a, s, st);
        return s.n == 3 ? aligned_only<T, 8, 3>(a, s, st) : aligned_only<T, 8, 8>(a, s, st);
    } else {
        if (s.n == 1) return by_alignment<T, 32, 1>(a, s, st);
        if (s.n == 4) return s.lt == 32 ? by_alignment<T, 32, 4>(a, s, st) : by_alignment<T, 8, 4>(a, s, st);
        return s.n == 3 ? by_alignment<T, 8, 3>(a, s, st) : s.n == 6 ? aligned_only<T, 8, 6>(a, s, st) : by_alignment<T, 8, 8>(a, s, st);
    }
}

int launch_block_tile_forward(const BlockArgs &a, int dtype, const TileShape &s, cudaStream_t st)
{
    return dtype == 0 ? by_shape<float>(a, s, st) : by_shape<bf16>(a, s, st);
}

}  // namespace hn
