// The residual block's backward on tiles (block.cu has the formulas).
//
// One meeting of the cluster a tile, for the three means of its tokens.  The sums over tokens that the weights' gradients are stay in
// registers over all tiles of a cluster; a slot of the workspace takes them at the end.
//
// 90 instructions an element with gate and dropout (values read again from shared memory and the gate worked out again behind the meeting,
// as registers for 16 warps an SM do not hold them) at 46 % of the issue slots; the barriers and the meeting take the rest.  16 x 4096 tokens
// of 768 channels, bf16: 274 us (0.45 of the measured copy rate), without dropout 241 (0.51); 884736 tokens of 64, fp32, no gate: 265
// (0.78).  The same overlap of tiles as in the forward: 296 us.
#include "block.cuh"

namespace hn {

namespace cg = cooperative_groups;

static __device__ int hn_block_status;                       // 1: a bounded wait gave up
int block_backward_status() { return read_status(hn_block_status); }

template <typename T, int LT, int N, bool ALIGNED> __global__ void __launch_bounds__(kTileThreads, N * (int)sizeof(T) > kBackwardBytes ? 1 : 2) block_tile_backward_kernel(BlockArgs p, int ctas)
{
    constexpr int TT = LT * V, ROWS = kTileThreads / LT;
    using Sums = TileSums<LT, 3>;
    using St = Stage<T, LT, N, 5, ALIGNED>;
    enum { X = 0, M = 1, Z = 2, DR = 3, DN = 4 };
    extern __shared__ __align__(16) char stages[];
    __shared__ Sums sums;
    __shared__ __align__(16) float rho[2][2][TT];                          // rho_m and rho_r of a tile's tokens
    pdl_join();
    int rank = 0;
    sums.init();
    if (LT == 8 && ctas > 1) {
        rank = cg::this_cluster().block_rank();
        cg::this_cluster().sync();
    }
    const bool drop = p.drop.threshold != 0;
    const DropKey key(drop ? DropKey(p.drop) : DropKey());
    const int row = threadIdx.x / LT, tl = threadIdx.x % LT, share = (p.C + ctas - 1) / ctas, c0 = rank * share + row;
    const int mine = min(share, p.C - rank * share);         // channels of this CTA
    const long long elements = (long long)p.B * p.C * p.T;
    const float D = drop ? p.drop.scale : 1.f;
    float w[N], gn[N], acc[N][2];                            // scale g_post / (1 - p); g_pre; sums over tokens
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int c = c0 + j * ROWS;
        const bool have = j * ROWS + row < mine;
        w[j] = D; gn[j] = acc[j][0] = acc[j][1] = 0.f;
        if (have && p.g_post) { HN_G(p.g_post + c, 4); w[j] *= __ldg(p.g_post + c); }
        if (have && p.scale) { HN_G(p.scale + c, 4); w[j] *= __ldg(p.scale + c); }
        if (have && p.g_pre) { HN_G(p.g_pre + c, 4); gn[j] = __ldg(p.g_pre + c); }
    }
    const long long entry = (long long)p.C * p.T, first = (long long)c0 * p.T, hop = (long long)ROWS * p.T;
    auto fetch = [&](char *stage, float (*to)[TT], const TileWalk &at) {
        if (at.inside(p.B)) {
            const int t0 = at.r * TT;
            St::fetch(stage, at.b * entry + (long long)rank * share * p.T + t0, p.T, mine, p.T - t0, elements, [&](auto piece) {
                piece(M, p.m);
                if (p.z) piece(Z, p.z);
                if (p.dn) { piece(X, p.x); piece(DN, p.dn); }
                if (p.dr) piece(DR, p.dr);
            });
            for (int i = threadIdx.x; i < 2 * TT; i += kTileThreads) {
                const int k = i / TT, t = t0 + i % TT;
                const bool wanted = t < p.T && (k ? p.g_pre : p.g_post);
                const float *src = p.stats + ((long long)k * p.B + at.b) * p.T + t;
                if (wanted) HN_G(src, 4);
                if (wanted) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"((unsigned)__cvta_generic_to_shared(&to[k][i % TT])), "l"(src) : "memory");
                else to[k][i % TT] = k ? 0.f : 1.f;
            }
        }
        stage_commit();
    };
    TileWalk here(blockIdx.x / ctas, gridDim.x / ctas, p.tiles_b), ahead = here;
    fetch(stages, rho[0], ahead);
    int meeting = 0;
    for (int turn = 0; here.inside(p.B); here.next(), turn ^= 1, ++meeting) {
        char *stage = stages + turn * St::BYTES;
        stage_wait<0>();
        __syncthreads();                                     // this tile and its rho are here, and the other stage has been read
        ahead.next();
        fetch(stages + (turn ^ 1) * St::BYTES, rho[turn ^ 1], ahead);
        const int t0 = here.r * TT, t = t0 + tl * V, count = p.T - t;
        const long long row0 = here.b * entry + first + t0;
        auto tokens = [&](const float *v, f2 (&f)[P]) {
            const float4 w = *reinterpret_cast<const float4 *>(v + tl * V);
            f[0] = make2(w.x, w.y); f[1] = make2(w.z, w.w);
        };
        f2 rm[P], rr[P], c1[P], c2[P];
        tokens(rho[turn][0], rm);
        tokens(rho[turn][1], rr);
        unsigned keep[N];
        if (drop) keep_bits<N>(key, p.T % 8 == 0, row0 + tl * V, hop, keep);
        // rho is kept out of the sums over channels: with k = scale D g_post act m,  x + rho_m k is r,  and with n' = rho_r dn,
        //     e r^ = g_pre n' r,     kappa (dr + rho_r e) = rho_m k (dr + g_pre n'),     kappa r^ = rho_m rho_r k r
        f2 s[3][P];
#pragma unroll
        for (int e = 0; e < P; ++e) s[0][e] = s[1][e] = s[2][e] = pair(0.f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const long long start = row0 + j * hop;
            f2 f[P], k[P];
            St::get(stage, M, j, start, count, k);
#pragma unroll
            for (int e = 0; e < P; ++e) k[e] = mul2(k[e], pair(w[j]));
            if (p.z) {
                f2 a[P], da[P];
                St::get(stage, Z, j, start, count, f);
                gates<false>(p.gate, f, a, da);
#pragma unroll
                for (int e = 0; e < P; ++e) k[e] = mul2(k[e], a[e]);
            }
            if (drop) drop_pairs(keep[j], k);
            if (p.dr) St::get(stage, DR, j, start, count, f);
            else f[0] = f[1] = pair(0.f);
            if (p.dn) {
                f2 n[P], r[P], local = pair(0.f);
                St::get(stage, DN, j, start, count, n);
                St::get(stage, X, j, start, count, r);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    r[e] = fma2(rm[e], k[e], r[e]);
                    n[e] = mul2(n[e], rr[e]);
                    local = fma2(n[e], r[e], local);
                    n[e] = mul2(n[e], pair(gn[j]));
                    s[0][e] = fma2(n[e], r[e], s[0][e]);
                    s[2][e] = fma2(k[e], r[e], s[2][e]);
                    f[e] = add2(f[e], n[e]);
                }
                acc[j][1] += sum2(local);
            }
#pragma unroll
            for (int e = 0; e < P; ++e) s[1][e] = fma2(k[e], f[e], s[1][e]);
        }
        const float inv = 1.f / (float)p.C;
        sums.sum(s, ctas, rank, meeting & 1, meeting >> 1 & 1, [&](int k, const float (&a)[3]) {
            const float om = rho[turn][0][k], on = rho[turn][1][k], mean = a[0] * inv;
            sums.total[0][k] = -on * on * mean;                                    // d = dr + g_pre n' - rho_r^2 c1 r
            sums.total[1][k] = -om * om * (om * (a[1] - on * on * mean * a[2]) * inv);     // dm = rho_m (f - m^ c2)
        });
        __syncthreads();
        if (sums.failed) break;
        tokens(sums.total[0], c1);
        tokens(sums.total[1], c2);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (j * ROWS + row >= mine || count <= 0) continue;
            const long long start = row0 + j * hop, i = start + tl * V;
            f2 m[P], a[P], da[P], d[P], am[P], local = pair(0.f);
            St::get(stage, M, j, start, count, m);
            if (p.z) {
                St::get(stage, Z, j, start, count, d);
                gates<true>(p.gate, d, a, da);
#pragma unroll
                for (int e = 0; e < P; ++e) am[e] = mul2(a[e], m[e]);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) am[e] = m[e];
            }
            if (drop) drop_pairs(keep[j], am);               // (nothing may come of what was dropped, not even 0 times infinity)
            if (p.dr) St::get(stage, DR, j, start, count, d);
            else d[0] = d[1] = pair(0.f);
            if (p.dn) {
                f2 n[P], r[P], k[P];
                St::get(stage, DN, j, start, count, n);
                St::get(stage, X, j, start, count, r);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    k[e] = mul2(am[e], pair(w[j]));
                    r[e] = fma2(rm[e], k[e], r[e]);
                    d[e] = fma2(mul2(n[e], rr[e]), pair(gn[j]), d[e]);
                    d[e] = fma2(r[e], c1[e], d[e]);
                }
            }
            st_vector<T, ALIGNED>(p.dx, i, count, d);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                f2 q = mul2(d[e], rm[e]);
                local = fma2(q, am[e], local);               // sum of keep d act m^: dg_post and dscale but for their constants
                q = mul2(q, pair(w[j]));
                if (p.z) {
                    da[e] = mul2(mul2(q, m[e]), da[e]);
                    q = mul2(q, a[e]);
                    if (drop) drop_pair(keep[j], e, da[e]);
                }
                if (drop) drop_pair(keep[j], e, q);
                d[e] = p.g_post ? fma2(m[e], c2[e], q) : q;
            }
            acc[j][0] += sum2(local);
            st_vector<T, ALIGNED>(p.dm, i, count, d);
            if (p.z) st_vector<T, ALIGNED>(p.dz, i, count, da);
        }
    }
    stage_wait<0>();
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
        for (int o = 1; o < LT; o *= 2) {
            acc[j][0] += __shfl_xor_sync(~0u, acc[j][0], o);
            acc[j][1] += __shfl_xor_sync(~0u, acc[j][1], o);
        }
        if (tl == 0 && j * ROWS + row < mine) {
            const int c = c0 + j * ROWS;
            float sc = D, gp = D;
            if (p.scale) { HN_G(p.scale + c, 4); sc *= __ldg(p.scale + c); }
            if (p.g_post) { HN_G(p.g_post + c, 4); gp *= __ldg(p.g_post + c); }
            float *q = p.partial + (long long)(blockIdx.x / ctas) * 3 * p.C + c;
            HN_G(q, 4); HN_G(q + p.C, 4); HN_G(q + 2 * p.C, 4);
            q[0] = sc * acc[j][0];
            q[p.C] = gp * acc[j][0];
            q[2 * p.C] = acc[j][1];
        }
    }
    if (LT == 8 && ctas > 1) {
        if (sums.failed && threadIdx.x == 0) atomicExch(&hn_block_status, 1);
        cg::this_cluster().sync();
    }
}

template <typename T, int LT, int N, bool ALIGNED> static int go(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    constexpr int BYTES = Stage<T, LT, N, 5, ALIGNED>::BYTES;
    return launch_tiles<block_tile_backward_kernel<T, LT, N, ALIGNED>, 2 * BYTES>(a, s, st);
}
template <typename T, int LT, int N> static int by_alignment(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    return a.T % (16 / sizeof(T)) == 0 ? go<T, LT, N, true>(a, s, st) : go<T, LT, N, false>(a, s, st);
}
template <typename T> static int by_shape(const BlockArgs &a, const TileShape &s, cudaStream_t st)
{
    constexpr int MOST = kBackwardBytes / (int)sizeof(T);
    if (s.n == 1 && s.lt == 32) return by_alignment<T, 32, 1>(a, s, st);
    if constexpr (sizeof(T) == 4) if (s.n == 1) return by_alignment<T, 8, 1>(a, s, st);
    if (s.n == 2) return s.lt == 32 ? by_alignment<T, 32, 2>(a, s, st) : by_alignment<T, 8, 2>(a, s, st);
    if constexpr (MOST >= 4) if (s.lt == 32) return by_alignment<T, 32, 4>(a, s, st);
    if constexpr (MOST >= 4) if (s.n == 3) return by_alignment<T, 8, 3>(a, s, st);
    if (s.n == 4) return by_alignment<T, 8, 4>(a, s, st);
    if constexpr (MOST >= 4) if (s.n == 8) return by_alignment<T, 8, 8>(a, s, st);
    return kNoLaunch;
}

int launch_block_tile_backward(const BlockArgs &a, int dtype, const TileShape &s, cudaStream_t st)
{
    return dtype == 0 ? by_shape<float>(a, s, st) : by_shape<bf16>(a, s, st);
}

}  // namespace hn
