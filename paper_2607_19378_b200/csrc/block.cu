// What stands between two mixers of a residual stream, for tensors [B][C][T] (T tokens, channels T elements apart):
//
//     w = act(z) * m rho_m g_post      rho_m = 1 / sqrt(mean_c m^2 + eps)       (norm of the mixer's output, gate)
//     r = x + scale * D * w            D = keep / (1 - p)                       (dropout, residual scale)
//     n = r rho_r g_pre                rho_r = 1 / sqrt(mean_c r^2 + eps)       (norm in front of the next mixer)
//
// and its gradient.  With e = g_pre dn, r^ = r rho_r, m^ = m rho_m, kappa = scale D act(z) g_post m^:
//
//     d  = dr + rho_r (e - r^ c1)      c1 = mean_c e r^          = dx
//     dz = scale D d m^ g_post act'(z);     f = scale D d act(z) g_post;     dm = rho_m (f - m^ c2),   c2 = mean_c f m^
//     dscale = sum d D w;     dg_post = sum scale D d act(z) m^;     dg_pre = sum dn r^
//
// f m^ = kappa d, so c2 = mean_c kappa (dr + rho_r e) - rho_r c1 mean_c kappa r^: both means of a token come from one walk over its
// channels.  The backward reads what the forward read and recomputes the rest; only the two rho of a token are kept.
//
// The kernels here take any number of channels: a CTA takes a tile of neighbouring tokens, its warps share the channels, and what a second
// walk needs is read again (from the caches, where it still is): 4096 tokens of 5000 channels, bf16, 234 and 470 us, 0.13 and 0.11 of the
// measured copy rate, latency of dependent loads.  Up to 2048 channels (1024 of fp32 forward where rows are no multiple of 16 bytes, and
// backward) tiles stay in shared memory (block_fwd.cu, block_bwd.cu): 2048 channels 35 and 77 us, 2100 here 90 and 212.
#include "block.cuh"

namespace hn {

// V neighbouring tokens of one channel (V = 4 only where 4 divides T)
template <typename T, int V> __device__ __forceinline__ void ld_tokens(const void *p, long long i, float (&f)[V])
{
    if constexpr (V == 1) f[0] = IO<T>::ld((const T *)p, i);
    else if constexpr (sizeof(T) == 4) {
        HN_G((const T *)p + i, 16);
        const float4 v = __ldg(reinterpret_cast<const float4 *>((const T *)p + i));
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
        HN_G((const T *)p + i, 8);
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>((const T *)p + i));
        unpack2(v.x, f[0], f[1]); unpack2(v.y, f[2], f[3]);
    }
}
template <typename T, int V> __device__ __forceinline__ void st_tokens(void *p, long long i, const float (&f)[V])
{
    if constexpr (V == 1) IO<T>::st((T *)p, i, f[0]);
    else if constexpr (sizeof(T) == 4) {
        HN_G((T *)p + i, 16);
        *reinterpret_cast<float4 *>((T *)p + i) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        HN_G((T *)p + i, 8);
        *reinterpret_cast<uint2 *>((T *)p + i) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
    }
}

// What one channel of V tokens contributes: gate, its slope, dropout factor, normalised mixer output
template <int V> struct Branch { float act[V], slope[V], D[V], mh[V], gp, sc; };

template <typename T, int V>
__device__ __forceinline__ void branch_of(const BlockArgs &p, const DropKey *key, long long i, int c, const float (&m)[V], const float (&rho)[V], Branch<V> &o)
{
    float z[V];
    if (p.z) ld_tokens<T, V>(p.z, i, z);
    o.gp = 1.f; o.sc = 1.f;
    if (p.g_post) { HN_G(p.g_post + c, 4); o.gp = __ldg(p.g_post + c); }
    if (p.scale) { HN_G(p.scale + c, 4); o.sc = __ldg(p.scale + c); }
    unsigned keep = ~0u;
    if (key) keep = key->keep(i >> 3) >> (i & 7);
    const bool silu = p.gate == GATE_SILU;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        o.act[e] = 1.f; o.slope[e] = 0.f;
        if (p.z) {
            f2 s, st;                                        // sigmoid and its slope; z s and s + z s' without a branch between the loads
            gate_pair<false, true>(pair(z[e]), s, st);
            o.act[e] = silu ? z[e] * s.x : s.x;
            o.slope[e] = silu ? fmaf(z[e], st.x, s.x) : st.x;
        }
        o.D[e] = key ? (keep >> e & 1 ? p.drop.scale : 0.f) : 1.f;
        o.mh[e] = m[e] * rho[e];
    }
}

// warps of a CTA: many where a lane has one token, so that few tokens of many channels keep the GPU busy
template <int V> constexpr int kBlockWarps = V == 1 ? 32 : 16;

// sums[k][e] over the CTA's warps, for this lane's tokens
template <int K, int V> __device__ __forceinline__ void sum_warps(float (&s)[K][V], float (*red)[K * 32 * V])
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    __syncthreads();                                         // the previous sums have been read
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) red[w][(k * V + e) * 32 + lane] = s[k][e];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float a = 0.f;
#pragma unroll
            for (int j = 0; j < kBlockWarps<V>; ++j) a += red[j][(k * V + e) * 32 + lane];
            s[k][e] = a;
        }
}

template <typename T, int V> __global__ void __launch_bounds__(kBlockWarps<V> * 32) block_forward_kernel(BlockArgs p)
{
    __shared__ float red[kBlockWarps<V>][32 * V];
    pdl_join();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const bool drop = p.drop.rng && p.drop.threshold;
    const DropKey key(drop ? DropKey(p.drop) : DropKey());
    const int b = (int)(blockIdx.x / p.tiles_b), t = (int)(blockIdx.x % p.tiles_b) * 32 * V + lane * V;
    const bool live = t < p.T;
    const long long base = (long long)b * p.C * p.T + t;
    float rho[V], s[1][V];
#pragma unroll
    for (int e = 0; e < V; ++e) { rho[e] = 1.f; s[0][e] = 0.f; }
    if (p.g_post) {
        if (live)
#pragma unroll 4
            for (int c = w; c < p.C; c += kBlockWarps<V>) {
                float m[V];
                ld_tokens<T, V>(p.m, base + (long long)c * p.T, m);
#pragma unroll
                for (int e = 0; e < V; ++e) s[0][e] = fmaf(m[e], m[e], s[0][e]);
            }
        sum_warps<1, V>(s, red);
#pragma unroll
        for (int e = 0; e < V; ++e) { rho[e] = rsqrtf(s[0][e] / (float)p.C + p.eps); s[0][e] = 0.f; }
    }
    auto value = [&](int c, float (&r)[V]) {
        const long long i = base + (long long)c * p.T;
        float m[V];
        Branch<V> o;
        ld_tokens<T, V>(p.m, i, m);
        ld_tokens<T, V>(p.x, i, r);
        branch_of<T, V>(p, drop ? &key : nullptr, i, c, m, rho, o);
#pragma unroll
        for (int e = 0; e < V; ++e) r[e] += o.D[e] != 0.f ? o.sc * (o.D[e] * (o.act[e] * (o.mh[e] * o.gp))) : 0.f;
    };
    if (live)
#pragma unroll 4
        for (int c = w; c < p.C; c += kBlockWarps<V>) {
            float r[V];
            value(c, r);
            st_tokens<T, V>(p.r, base + (long long)c * p.T, r);
#pragma unroll
            for (int e = 0; e < V; ++e) s[0][e] = fmaf(r[e], r[e], s[0][e]);
        }
    float rho_r[V];
    if (p.g_pre) {
        sum_warps<1, V>(s, red);
#pragma unroll
        for (int e = 0; e < V; ++e) rho_r[e] = rsqrtf(s[0][e] / (float)p.C + p.eps);
        if (live)
#pragma unroll 4
            for (int c = w; c < p.C; c += kBlockWarps<V>) {
                float r[V];
                value(c, r);
                HN_G(p.g_pre + c, 4);
                const float g = __ldg(p.g_pre + c);
#pragma unroll
                for (int e = 0; e < V; ++e) r[e] *= rho_r[e] * g;
                st_tokens<T, V>(p.n, base + (long long)c * p.T, r);
            }
    }
    if (p.stats && live && w == 0) {
        if (p.g_post) st_tokens<float, V>(p.stats, (long long)b * p.T + t, rho);
        if (p.g_pre) st_tokens<float, V>(p.stats, ((long long)p.B + b) * p.T + t, rho_r);
    }
}

template <typename T, int V> __global__ void __launch_bounds__(kBlockWarps<V> * 32) block_backward_kernel(BlockArgs p)
{
    __shared__ float red[kBlockWarps<V>][3 * 32 * V];
    pdl_join();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const bool drop = p.drop.rng && p.drop.threshold;
    const DropKey key(drop ? DropKey(p.drop) : DropKey());
    float *slot = p.partial + (long long)blockIdx.x * 3 * p.C;
    bool first = true;
    for (long long tile = blockIdx.x; tile < p.tiles; tile += gridDim.x, first = false) {
        const int b = (int)(tile / p.tiles_b), t = (int)(tile % p.tiles_b) * 32 * V + lane * V;
        const bool live = t < p.T;
        const long long base = (long long)b * p.C * p.T + t;
        float rho_m[V], rho_r[V], s[3][V];
#pragma unroll
        for (int e = 0; e < V; ++e) { rho_m[e] = 1.f; rho_r[e] = 0.f; s[0][e] = s[1][e] = s[2][e] = 0.f; }
        if (live && p.g_post) ld_tokens<float, V>(p.stats, (long long)b * p.T + t, rho_m);
        if (live && p.g_pre) ld_tokens<float, V>(p.stats, ((long long)p.B + b) * p.T + t, rho_r);
        // of one channel: gradient of n times g_pre, r^, gradient of r
        auto values = [&](int c, Branch<V> &o, float (&en)[V], float (&rh)[V], float (&dr)[V], float &g) {
            const long long i = base + (long long)c * p.T;
            float m[V], x[V];
            ld_tokens<T, V>(p.m, i, m);
            branch_of<T, V>(p, drop ? &key : nullptr, i, c, m, rho_m, o);
#pragma unroll
            for (int e = 0; e < V; ++e) { en[e] = rh[e] = dr[e] = 0.f; }
            g = 0.f;
            if (p.dr) ld_tokens<T, V>(p.dr, i, dr);
            if (p.g_pre) {
                ld_tokens<T, V>(p.dn, i, en);
                ld_tokens<T, V>(p.x, i, x);
                HN_G(p.g_pre + c, 4);
                g = __ldg(p.g_pre + c);
#pragma unroll
                for (int e = 0; e < V; ++e) rh[e] = (x[e] + (o.D[e] != 0.f ? o.sc * (o.D[e] * (o.act[e] * (o.mh[e] * o.gp))) : 0.f)) * rho_r[e];
            }
        };
        if (live && (p.g_pre || p.g_post))
#pragma unroll 4
            for (int c = w; c < p.C; c += kBlockWarps<V>) {
                Branch<V> o;
                float en[V], rh[V], dr[V], g;
                values(c, o, en, rh, dr, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float kappa = o.D[e] != 0.f ? o.sc * o.D[e] * o.act[e] * o.gp * o.mh[e] : 0.f, eg = en[e] * g;
                    s[0][e] = fmaf(eg, rh[e], s[0][e]);
                    s[1][e] = fmaf(kappa, fmaf(rho_r[e], eg, dr[e]), s[1][e]);
                    s[2][e] = fmaf(kappa, rh[e], s[2][e]);
                }
            }
        sum_warps<3, V>(s, red);
        float c1[V], c2[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            c1[e] = s[0][e] / (float)p.C;
            c2[e] = p.g_post ? (s[1][e] - rho_r[e] * c1[e] * s[2][e]) / (float)p.C : 0.f;
        }
#pragma unroll 2
        for (int c = w; c < p.C; c += kBlockWarps<V>) {
            float sum[3] = {0.f, 0.f, 0.f};
            if (live) {
                Branch<V> o;
                float en[V], rh[V], dr[V], g, d[V], dm[V], dz[V];
                values(c, o, en, rh, dr, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    d[e] = dr[e] + rho_r[e] * (en[e] * g - rh[e] * c1[e]);
                    const bool kept = o.D[e] != 0.f;
                    const float mn = o.mh[e] * o.gp, dD = kept ? d[e] * o.D[e] : 0.f, dw = o.sc * dD, df = kept ? dw * o.act[e] : 0.f;
                    dz[e] = kept ? dw * mn * o.slope[e] : 0.f;
                    sum[0] += kept ? df * o.mh[e] : 0.f;
                    sum[1] += kept ? dD * (o.act[e] * mn) : 0.f;
                    sum[2] = fmaf(en[e], rh[e], sum[2]);
                    dm[e] = p.g_post ? rho_m[e] * (df * o.gp - o.mh[e] * c2[e]) : df;
                }
                const long long i = base + (long long)c * p.T;
                st_tokens<T, V>(p.dx, i, d);
                st_tokens<T, V>(p.dm, i, dm);
                if (p.z) st_tokens<T, V>(p.dz, i, dz);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int o = 16; o; o /= 2) sum[k] += __shfl_xor_sync(~0u, sum[k], o);
            if (lane < 3) {
                float *q = slot + (long long)lane * p.C + c;
                const float v = lane == 0 ? sum[0] : lane == 1 ? sum[1] : sum[2];
                HN_G(q, 4);
                *q = first ? v : *q + v;
            }
        }
    }
}

// out[k][c] = sum of the slots, a fixed order whatever the timing: 32 chains a channel, four loads of each on their way, then those
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(kSumWarps * 32) block_sum_kernel(const float *partial, int slots, int C, float *dg_post, float *dscale, float *dg_pre)
{
    __shared__ float red[kSumWarps][33];
    pdl_join();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (i < 3 * C)
        for (int j = w; j < slots; j += 4 * kSumWarps) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *q = partial + (long long)(j + u * kSumWarps) * 3 * C + i;
                v[u] = 0.f;
                if (j + u * kSumWarps < slots) { HN_G(q, 4); v[u] = *q; }
            }
            s += (v[0] + v[1]) + (v[2] + v[3]);
        }
    red[w][lane] = s;
    __syncthreads();
    s = red[lane][w];                                        // warp w: the block's channel w
#pragma unroll
    for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
    const int c = blockIdx.x * 32 + w;
    if (lane || c >= 3 * C) return;
    float *out = c < C ? dg_post : c < 2 * C ? dscale : dg_pre;
    if (out) { HN_G(out + c % C, 4); out[c % C] = s; }
}

// How the tile kernels take a shape: few channels in one CTA with wide tiles of tokens, more in a cluster, at two CTAs an SM; twice as
// many channels at one CTA an SM (backward, 4 x 64 x 64 tokens of 768 channels, fp32: 103 us, the general kernels 347).  false: more
// channels than a cluster holds.
static bool tile_shape(const BlockArgs &a, int dtype, bool backward, TileShape *s)
{
    const bool ragged = a.T * elsize(dtype) % 16 != 0;
    int most = (backward ? kBackwardBytes : kForwardBytes) / (int)elsize(dtype);       // channels of a thread
    if (!backward && ragged && a.C <= kTileCtas * 16 * most) most /= 2;                // (rows with a piece more: two CTAs an SM all the same)
    s->lt = a.C <= 8 * (most < 4 ? most : 4) ? 32 : 8;
    const int rows = kTileThreads / s->lt;
    if (a.C > kTileCtas * rows * most) {
        if (!backward && ragged && dtype == HYENAND_F32) return false;                 // (would not fit in an SM's shared memory)
        most *= 2;
    }
    s->ctas = (a.C + rows * most - 1) / (rows * most);
    if (s->ctas > kTileCtas || most > 8) return false;
    const int each = ((a.C + s->ctas - 1) / s->ctas + rows - 1) / rows;
    // (widths of 96, 192, 384: 16 x 4096 tokens of 192 channels, bf16, dropout: forward with six 37 us, with eight 45; backward with three 79, with four 83)
    s->n = each <= 2 ? each : each == 3 && s->lt == 8 ? 3 : each <= 4 ? 4 : each <= 6 && !backward ? 6 : 8;
    return true;
}

// workspace slots written, or below 0 (finish)
static int block_launch(BlockArgs &a, int dtype, bool backward, cudaStream_t st)
{
    TileShape s{};
    if (tile_shape(a, dtype, backward, &s)) {
        const int tokens = s.lt * V;
        a.tiles_b = (a.T + tokens - 1) / tokens;
        a.tiles = (long long)a.B * a.tiles_b;
        return (backward ? launch_block_tile_backward : launch_block_tile_forward)(a, dtype, s, st);
    }
    const int tokens = a.T % 4 == 0 && (long long)a.B * ((a.T + 127) / 128) >= kSms ? 4 : 1;
    a.tiles_b = (a.T + 32 * tokens - 1) / (32 * tokens);
    a.tiles = (long long)a.B * a.tiles_b;
    const long long blocks = backward && a.tiles > kBlockSlots ? kBlockSlots : a.tiles;
    if (blocks > 0x7fffffffll) return kTooLarge;
#define HN_BLK(T, V) launch_pdl(backward ? block_backward_kernel<T, V> : block_forward_kernel<T, V>, dim3((unsigned)blocks), kBlockWarps<V> * 32, 0, st, a)
    if (dtype == HYENAND_F32) { if (tokens == 4) HN_BLK(float, 4); else HN_BLK(float, 1); }
    else { if (tokens == 4) HN_BLK(bf16, 4); else HN_BLK(bf16, 1); }
#undef HN_BLK
    return (int)blocks;
}

static int check_block(int B, int C, int T, int dtype, const void *x, const void *m, const void *z, const float *g_pre, float eps, int gate, float p,
                       const long long *rng, int site, BlockArgs *a)
{
    if (B < 1 || C < 1 || T < 1) return fail(HYENAND_ERR_INVALID_ARG, "B, C and T must be >= 1");
    if (T > (1 << 30) || C > (1 << 20) || (long long)B * T > (1ll << 40) / C)
        return fail(HYENAND_ERR_UNSUPPORTED, "T is above 2^30, C above 2^20 or B C T above 2^40");
    if (dtype != HYENAND_F32 && dtype != HYENAND_BF16) return fail(HYENAND_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (gate < GATE_NONE || gate > GATE_SILU) return fail(HYENAND_ERR_INVALID_ARG, "unknown gate %d", gate);
    if (!x || !m) return fail(HYENAND_ERR_INVALID_ARG, "x and m must be non-NULL");
    if ((z != nullptr) != (gate != GATE_NONE)) return fail(HYENAND_ERR_INVALID_ARG, "z is given with a gate and only with one");
    if (!(eps > 0.f) || eps > 1e30f) return fail(HYENAND_ERR_INVALID_ARG, "eps must be positive and finite");
    if (!drop_args(p, rng, site, &a->drop)) return fail(HYENAND_ERR_INVALID_ARG, "p must be in [0, 1)");
    if (a->drop.threshold && !rng) return fail(HYENAND_ERR_INVALID_ARG, "rng must be non-NULL where p > 0");
    a->x = x; a->m = m; a->z = z; a->g_pre = g_pre; a->eps = eps; a->gate = gate; a->B = B; a->C = C; a->T = T;
    return HYENAND_OK;
}

static void block_inputs(CallTensors &c, const BlockArgs &a, size_t nb)
{
    const size_t wb = (size_t)a.C * sizeof(float);
    c.in("x", a.x, nb); c.in("m", a.m, nb); c.in("z", a.z, nb);
    c.in("g_post", a.g_post, wb, 4); c.in("scale", a.scale, wb, 4); c.in("g_pre", a.g_pre, wb, 4);
    if (a.drop.threshold) c.in("rng", a.drop.rng, 2 * sizeof(long long));
}

}  // namespace hn

using namespace hn;

extern "C" int hyenand_block_forward(int B, int C, int T, int dtype, const void *x, const void *m, const void *z, const float *g_post,
                                     const float *scale, const float *g_pre, float eps, int gate, float p, const long long *rng, int site,
                                     void *r, void *n, float *stats, void *cuda_stream)
{
    clear_error();
    BlockArgs a{};
    if (int e = check_block(B, C, T, dtype, x, m, z, g_pre, eps, gate, p, rng, site, &a)) return e;
    if (!r) return fail(HYENAND_ERR_INVALID_ARG, "r must be non-NULL");
    if ((n != nullptr) != (g_pre != nullptr)) return fail(HYENAND_ERR_INVALID_ARG, "n is given with g_pre and only with it");
    a.g_post = g_post; a.scale = scale; a.r = r; a.n = n; a.stats = stats;
    CallTensors c;
    const size_t nb = (size_t)B * C * T * elsize(dtype);
    block_inputs(c, a, nb);
    c.out("r", r, nb); c.out("n", n, nb); c.out("stats", stats, (size_t)2 * B * T * sizeof(float));
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(block_launch(a, dtype, false, (cudaStream_t)cuda_stream));
}

extern "C" long long hyenand_block_workspace_bytes(int B, int C, int T, int dtype)
{
    (void)dtype;
    if (B < 1 || C < 1 || T < 1) return 0;
    const long long tiles = (long long)B * (((long long)T + 31) / 32);       // (no kernel's are smaller)
    return (tiles < kBlockSlots ? tiles : kBlockSlots) * 3 * C * (long long)sizeof(float);
}

extern "C" int hyenand_block_device_status(void)
{
    if (cudaDeviceSynchronize() != cudaSuccess) return -1;
    const int f = block_forward_status(), b = block_backward_status();
    return f < 0 || b < 0 ? -1 : f | b;
}

extern "C" int hyenand_block_backward(int B, int C, int T, int dtype, const void *x, const void *m, const void *z, const float *g_post,
                                      const float *scale, const float *g_pre, float eps, int gate, float p, const long long *rng, int site,
                                      const float *stats, const void *dr, const void *dn, void *dx, void *dm, void *dz, float *dg_post,
                                      float *dscale, float *dg_pre, void *workspace, void *cuda_stream)
{
    clear_error();
    BlockArgs a{};
    if (int e = check_block(B, C, T, dtype, x, m, z, g_pre, eps, gate, p, rng, site, &a)) return e;
    if (!dx || !dm || !workspace) return fail(HYENAND_ERR_INVALID_ARG, "dx, dm and workspace must be non-NULL");
    if ((dz != nullptr) != (z != nullptr)) return fail(HYENAND_ERR_INVALID_ARG, "dz is given with z and only with it");
    if ((dn != nullptr) != (g_pre != nullptr)) return fail(HYENAND_ERR_INVALID_ARG, "dn is given with g_pre and only with it");
    if (!dr && !dn) return fail(HYENAND_ERR_INVALID_ARG, "dr or dn must be given");
    if ((g_post || g_pre) && !stats) return fail(HYENAND_ERR_INVALID_ARG, "stats must be non-NULL where a norm is");
    if ((dg_post && !g_post) || (dscale && !scale) || (dg_pre && !g_pre)) return fail(HYENAND_ERR_INVALID_ARG, "a gradient is asked of a weight that is not given");
    a.g_post = g_post; a.scale = scale; a.stats = (float *)stats; a.dr = dr; a.dn = dn; a.dx = dx; a.dm = dm; a.dz = dz;
    a.partial = (float *)workspace;
    CallTensors c;
    const size_t nb = (size_t)B * C * T * elsize(dtype), wb = (size_t)C * sizeof(float);
    block_inputs(c, a, nb);
    if (g_post || g_pre) c.in("stats", stats, (size_t)2 * B * T * sizeof(float));
    c.in("dr", dr, nb); c.in("dn", dn, nb);
    c.out("dx", dx, nb); c.out("dm", dm, nb); c.out("dz", dz, nb);
    c.out("dg_post", dg_post, wb, 4); c.out("dscale", dscale, wb, 4); c.out("dg_pre", dg_pre, wb, 4);
    c.out("workspace", workspace, (size_t)hyenand_block_workspace_bytes(B, C, T, dtype));
    if (int e = c.check()) return e;
    c.register_ranges();
    const int slots = block_launch(a, dtype, true, (cudaStream_t)cuda_stream);
    if (slots > 0 && (dg_post || dscale || dg_pre))
        launch_pdl(block_sum_kernel, dim3((unsigned)((3ll * C + 31) / 32)), kSumWarps * 32, 0, (cudaStream_t)cuda_stream, (const float *)a.partial, slots, C, dg_post, dscale, dg_pre);
    return finish(slots);
}
