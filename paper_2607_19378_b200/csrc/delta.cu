// The gated delta rule: forward pass, in chunks (formulas and number formats in delta.cuh).
//
// prepare: a CTA per chunk and head, all at once: k k^T and q k^T as one product of 128 rows, decays, A in fp32 (blocks of 16 by
//     substitution, then merged in pairs), A and P as planes into the workspace.
// walk: a CTA per head walks its chunks.  The state's rows are the lanes of tensor memory (Dv of 128), so that S^T products chain without a
//     transposition: S k, then A Z, then the new state each take the result of the one before as their A operand in tensor memory, through
//     registers (256 threads: a lane's columns in two halves).  The fp32 state stays in registers.  One warp issues the products, three
//     fetch the next chunks, four take the results.
// Few heads and many chunks: the walk is serial, so a head is cut into segments.  Where a segment starts from nothing it gives N, where it
//     starts from the identity without values it gives Phi, and from any state S it ends at S Phi + N: both walks run for all
//     segments at once, a small kernel joins them, and the walk proper starts every segment at once.
#include <atomic>

#include "delta.cuh"

namespace hn {

static __device__ int hn_delta_status;

// ---- prepare --------------------------------------------------------------------------------------------------------

template <typename T, int KD> struct Prep {
    static constexpr int PI = Planes<T>::IN, PM = Planes<T>::MID, PA = Planes<T>::INVERSE, TILE = KD * 128, PITCH = 2 * TILE, TROW = 68;
    // the tiles of k and q; T and the planes of P take their place
    static constexpr int P = kTok * TROW * 4 + 1024 - kTok * TROW * 4 % 1024, AFTER = P + PM * kMatrix, IMAGES = PI * PITCH > AFTER ? PI * PITCH : AFTER, BYTES = 1024 + IMAGES;
};

// C = -A B for the lower left block of N x N of a pair of blocks, in place: rows r0 + N .., columns r0 ..; A = T's block, B = the upper
// inverse (first), or A = the lower inverse, B = C (then).  `threads` threads of a pair, each one row and N N / threads columns.
template <int N, int THREADS, bool FIRST> __device__ __forceinline__ void merge(float *T, int row, int r0, int t)
{
    constexpr int EACH = N * N / THREADS;                    // 4 or 8
    const int r = r0 + N + t / (N / EACH), c = r0 + t % (N / EACH) * EACH;
    f2 acc[EACH / 2];
#pragma unroll
    for (int e = 0; e < EACH / 2; ++e) acc[e] = pair(0.f);
    // first: sum over m of T[r][r0 + m] B[r0 + m][c]; then: of inverse[r][r0 + N + m] C[r0 + N + m][c]
    const float *left = T + r * row + (FIRST ? r0 : r0 + N), *right = T + (FIRST ? r0 : r0 + N) * row + c;
#pragma unroll 2
    for (int m = 0; m < N; m += 4) {
        const float4 l = *(const float4 *)(left + m);
        const float lm[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < EACH; e += 4) {
                const float4 w = *(const float4 *)(right + (m + i) * row + e);
                acc[e / 2] = fma2(pair(lm[i]), make2(w.x, w.y), acc[e / 2]);
                acc[e / 2 + 1] = fma2(pair(lm[i]), make2(w.z, w.w), acc[e / 2 + 1]);
            }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH / 2; e += 2) {
        const f2 p = FIRST ? acc[e] : mul2(acc[e], pair(-1.f)), q = FIRST ? acc[e + 1] : mul2(acc[e + 1], pair(-1.f));
        *(float4 *)(T + r * row + c + 2 * e) = make_float4(p.x, p.y, q.x, q.y);
    }
    __syncthreads();
}

// Read: a chunk's k and q; written: 24 KB of planes of A and 16 of P (bf16).  6144 chunks of 128 channels: 117 us, 0.41 GB, 3.5 TB/s.  It is
// bound by the latency of its steps one after the other (copy, product, inverse, stores), which the few CTAs that an SM holds only partly
// cover.  The inverse by blocks in place of 64 dependent steps took a batch of prompts, 192 heads of 64, from 319 to 230 us in all.
template <typename T, int KD> __global__ void __launch_bounds__(128) delta_prepare_kernel(DeltaArgs a, const __grid_constant__ DeltaMaps maps)
{
    using C = Prep<T, KD>;
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ __align__(16) float hi[kTok], lo[kTok], beta[kTok];
    __shared__ uint64_t bar, there;
    __shared__ unsigned slot;
    unsigned char *sm = align_images(raw);
    float *Ts = (float *)sm;
    const int tid = threadIdx.x, warp = uniform_warp(tid >> 5), lane = tid & 31;
    const long long at = blockIdx.x, bh = at / a.chunks;
    const int chunk = (int)(at % a.chunks), b = (int)(bh / a.H), h = (int)(bh % a.H), t0 = chunk * kTok;
    pdl_wait();
    const int n = live_tokens(a, b), nv = n - t0 < kTok ? n - t0 : kTok;
    if (nv <= 0) return;
    const long long bk = (long long)b * a.Hk + h / (a.H / a.Hk);
    const int steps = (a.Dk + 15) / 16;
    const bool copied = by_copy(a, nv, t0);
    if (tid == 0) {
        mbar_init(&bar, 1); mbar_init(&there, 1);
        fence_mbar_init();
        if (copied) {
            mbar_expect_tx(&there, 2 * C::TILE);
            tma_load_3d(sm, &maps.k, &there, t0, 0, (int)bk);
            tma_load_3d(sm + C::TILE, &maps.q, &there, t0, 0, (int)bk);
        }
    }
    __syncwarp();
    if (warp == 0) tmem_alloc(smem_u32(&slot), 64);
    if (!copied) {
        const long long qk = bk * a.Dk * a.L + t0, all = (long long)a.B * a.Hk * a.Dk * a.L;
        load_tile<T>(sm, C::PITCH, (const T *)a.k, qk, all, a.L, a.Dk, nv, tid, 128);
        load_tile<T>(sm + C::TILE, C::PITCH, (const T *)a.q, qk, all, a.L, a.Dk, nv, tid, 128);
        clear_rows(sm, C::PITCH, C::PI, a.Dk, steps * 16, tid, 128);
        clear_rows(sm + C::TILE, C::PITCH, C::PI, a.Dk, steps * 16, tid, 128);
    }
    const long long row = bh * a.L + t0;
    if (warp == 1) chunk_sums(hi, lo, a.g + row, a.decay, nv, lane);
    if (warp >= 2) {
        const int t = tid - 64;
        beta[t] = 0.f;
        if (t < nv) { HN_G(a.beta + row + t, 4); beta[t] = __ldg(a.beta + row + t); }
    }
    fence_async_smem();
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const unsigned tb = slot, images = smem_u32(sm);
    bool ok = (!copied || mbar_wait(&there, 0)) && !is_late(a, LATE_PREPARE, bh, chunk, LATE_COPIES);
    if (warp == 0) {
        issue_ss<C::PI, C::PI, C::PI, true, true, KD / 16>(tb, images, C::PITCH, C::TILE, images, C::PITCH, steps, kTok, false);
        umma_commit(&bar);
    }
    auto store_gates = [&](float sick) {                     // (of a token each; sick: 0, or NaN)
        float *gates = a.gates + at * kGates;
        const float gamma = ratio(hi[tid], lo[tid], 0.f, 0.f) + sick;
        const float x[6] = {gamma, ratio(hi[kTok - 1], lo[kTok - 1], hi[tid], lo[tid]) + sick, beta[tid] + sick, -beta[tid] * gamma, hi[tid] + sick, lo[tid] + sick};
#pragma unroll
        for (int e = 0; e < 6; ++e) {
            float *to = gates + (e < 4 ? 0 : kSums - kCarry) + e * kTok + tid;
            HN_G(to, 4);
            *to = x[e];
        }
        if (tid == kTok - 1) {                               // (its gamma is the chunk's)
            const float less = expm1f((hi[tid] + lo[tid]) * 0.6931471805599453f) + sick;
            HN_G(gates + kCarry, 16);
            *(float4 *)(gates + kCarry) = less > -0.5f ? make_float4(1.f, less, 0.f, 0.f) : make_float4(0.f, gamma, 0.f, 0.f);
        }
    };
    if (tid < kTok) store_gates(0.f);                        // (the decays meanwhile)
    ok = mbar_wait(&bar, 0) && ok && !is_late(a, LATE_PREPARE, bh, chunk, LATE_PRODUCT);
    tmem_fence_after_sync();
    if (__syncthreads_or(!ok)) {                             // (every thread has waited: the tiles' place is free)
        // the chunk's factors are NaN, and with them all that comes of it; copies and products under way end before the CTA does
        if (!ok) atomicExch(&hn_delta_status, 1);
        if (copied) mbar_wait(&there, 0);
        mbar_wait(&bar, 0);
        if (tid < kTok) store_gates(kLost);
    }
    // lanes 0 .. 63: rows of k k^T, lanes 64 .. 127: rows of q k^T
    const int i = tid & 63;
    {
        const float Hi = hi[i], Li = lo[i], bi = beta[i];
        const unsigned at_row = tmem_addr(tb, warp, 0);
#pragma unroll 2
        for (int g = 0; g < 8; ++g) {
            float x[8];
            if (g >= 4 && !(warp & 1)) {                      // rows 0 .. 31 have nothing there
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
            } else {
                tmem_ld8(x, at_row + 8 * g);
                tmem_wait_ld();
                const float4 h0 = *(const float4 *)(hi + 8 * g), h1 = *(const float4 *)(hi + 8 * g + 4), l0 = *(const float4 *)(lo + 8 * g), l1 = *(const float4 *)(lo + 8 * g + 4);
                const float hj[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w}, lj[8] = {l0.x, l0.y, l0.z, l0.w, l1.x, l1.y, l1.z, l1.w};
                // (a later token's ratio is of no use and may be no number)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = 8 * g + e;
                    x[e] *= ratio(Hi, Li, hj[e], lj[e]);
                    x[e] = warp < 2 ? (j < i ? bi * x[e] : 0.f) : (j <= i ? x[e] : 0.f);
                }
            }
            if (warp < 2) {
                *(float4 *)(Ts + i * C::TROW + 8 * g) = make_float4(x[0], x[1], x[2], x[3]);
                *(float4 *)(Ts + i * C::TROW + 8 * g + 4) = make_float4(x[4], x[5], x[6], x[7]);
            } else planes8_to_image<C::PM>(sm + C::P, kMatrix, i, g, x);
        }
    }
    fence_async_smem();
    tmem_fence_before_sync();
    __syncthreads();
    unsigned char *to = a.images + at * ((C::PA + C::PM) * kMatrix);
    if (tid == 96) {
        bulk_store(to + C::PA * kMatrix, sm + C::P, C::PM * kMatrix);
        tma_commit();
    }
    if (warp == 0) tmem_dealloc(tb, 64);
    pdl_trigger();                                           // (late: see delta.cuh)
    // A = (I + T)^{-1} in T's place: blocks of 16 by forward substitution, a thread a column; then pairs of blocks,
    //     (D1 0; T21 D2)^{-1} = (D1^{-1} 0; -D2^{-1} T21 D1^{-1} D2^{-1}), to 32 and to 64
    if (tid < kTok) {
        float *D = Ts + (tid & 48) * (C::TROW + 1);
        const int j = tid & 15;
        float c[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float s[2] = {r == j ? 1.f : 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < r; m += 4) {
                const float4 w = *(const float4 *)(D + r * C::TROW + m);
                s[0] = fmaf(-w.x, c[m], s[0]);
                if (m + 1 < r) s[1] = fmaf(-w.y, c[m + 1], s[1]);
                if (m + 2 < r) s[0] = fmaf(-w.z, c[m + 2], s[0]);
                if (m + 3 < r) s[1] = fmaf(-w.w, c[m + 3], s[1]);
            }
            c[r] = s[0] + s[1];
        }
        __syncwarp();                                         // (the block's columns are in one warp)
#pragma unroll
        for (int r = 0; r < 16; ++r) D[r * C::TROW + j] = c[r];
    }
    __syncthreads();
    merge<16, 64, true>(Ts, C::TROW, tid >> 6 << 5, tid & 63);
    merge<16, 64, false>(Ts, C::TROW, tid >> 6 << 5, tid & 63);
    merge<32, 128, true>(Ts, C::TROW, 0, tid);
    merge<32, 128, false>(Ts, C::TROW, 0, tid);
#pragma unroll 1
    for (int e = tid; e < kTok * 8; e += 128) {
        const int r = e >> 3, c = e & 7;
        const float4 u = *(const float4 *)(Ts + r * C::TROW + 8 * c), v = *(const float4 *)(Ts + r * C::TROW + 8 * c + 4);
        const float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
        uint4 w[C::PA];
        planes8<C::PA>(w, x);
#pragma unroll
        for (int p = 0; p < C::PA; ++p) {
            uint4 *o = (uint4 *)(to + p * kMatrix + image_at(r, c));
            HN_G(o, 16);
            *o = w[p];
        }
    }
    if (tid == 96) tma_wait_all0();
}

// ---- walk -----------------------------------------------------------------------------------------------------------

#define WAIT(bar, parity) walk_wait(&ws, bar, parity)

template <typename T, int KD> struct Walk {
    static constexpr int PI = Planes<T>::IN, PM = Planes<T>::MID, PA = Planes<T>::INVERSE, TILE = KD * 128, TENSOR = PI * TILE;
    static constexpr bool VALUES = PI == 1;                                   // values and results travel as images
    static constexpr int IMAGES = (PA + PM) * kMatrix, K = 0, Q = TENSOR, A = 2 * TENSOR, V = A + IMAGES, GATES = V + (VALUES ? TILE : 0), STAGE = GATES + kWalkGates;
    static constexpr int OUT = VALUES ? 2 * TILE : 0;                         // two images of results
    static constexpr int STAGES = 3 * STAGE + OUT <= kWalkBytes ? 3 : 2 * STAGE + OUT <= kWalkBytes ? 2 : 1;
    static constexpr int BYTES = STAGES * STAGE + OUT;
    // tensor memory: S as an operand | Z, later U, as an operand | S k, then U | S q, then y | what S gains | delta U as an operand
    static constexpr int SCOLS = PM * KD / 2, ZCOLS = PM * kTok / 2, S0 = 0, Z0 = SCOLS, X0 = Z0 + ZCOLS, Y0 = X0 + kTok;
    // (with three planes of 128 columns delta U takes S's place, and the first half of the gain U's)
    static constexpr bool ROOM = Y0 + kTok + KD + ZCOLS <= 512;
    static constexpr int D0 = ROOM ? Y0 + kTok : X0, D1 = ROOM ? D0 + KD / 2 : Y0 + kTok, U0 = ROOM ? D0 + KD : S0;
    static_assert((ROOM || (D1 + KD / 2 <= 512 && KD / 2 == kTok)) && BYTES <= kWalkBytes, "tensor and shared memory");
};

// Bound by the chain of a chunk: S k, Z, A Z, the new state, each a product (some 300 to 700 cycles with its issue and its end's way back)
// and a passage through registers (350 to 1300).  3.8 us a chunk of 128 channels (96 heads of 4096 tokens: 241 us), whatever
// the bytes: 0.5 GB, 2.3 TB/s.  What shortened it: y, its scaling and its stores on other warps (off the chain), the fp32 state in registers,
// the columns of S in two halves so that S k begins with the first, kept states stored in three parts (a quarter, a quarter, a half) while products run (265 -> 242), values read
// before the product they meet (242 -> 232).  Prefetches into L2 and more stages made it slower, as did anything that grew the code.
template <typename T, int KD, int MODE> __global__ void __launch_bounds__(kWalkThreads, 1) delta_walk_kernel(DeltaArgs a, const __grid_constant__ DeltaMaps maps)
{
    using C = Walk<T, KD>;
    constexpr int PI = C::PI, PM = C::PM, HC = KD / 2;
    constexpr bool RUN = MODE == WALK_RUN;
    constexpr int KERNEL = RUN ? LATE_WALK : LATE_MAPS;
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ WalkShared ws;
    unsigned char *const sm = raw;
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp(tid >> 5);
    long long id = blockIdx.x;
    const bool phi = !RUN && (id & 1);                       // from the identity, without values
    if (!RUN) id >>= 1;
    const long long bh = id / a.segments;
    const int segment = (int)(id % a.segments), b = (int)(bh / a.H), h = (int)(bh % a.H);
    pdl_wait();
    const int n = live_tokens(a, b), first = segment * a.per_segment, end = first + a.per_segment < a.chunks ? first + a.per_segment : a.chunks;
    int last = (n + kTok - 1) / kTok;                        // chunks first .. last - 1 hold tokens
    last = last < end ? last : end;
    if (warp == 0) tmem_alloc(smem_u32(&ws.slot), 512);
    if (tid == 0) {
        walk_init(&ws, C::STAGES);
        walk_late(&ws, smem_u32(raw) & 1023u);               // (images that start elsewhere would be read wrongly: see kWalkBytes)
    }
    for (int s = 0; s < C::STAGES; ++s) {
        clear_rows(sm + s * C::STAGE, C::TILE, 2 * PI, a.Dk, KD, tid, kWalkThreads);
        if (C::VALUES) clear_rows(sm + s * C::STAGE + C::V, C::TILE, 1, phi ? 0 : a.Dv, KD, tid, kWalkThreads);
    }
    fence_async_smem();
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const unsigned tb = ws.slot;
    const long long states = (long long)a.Dv * a.Dk, vhead = bh * a.Dv * a.L, vall = (long long)a.B * a.H * a.Dv * a.L;
    if (warp > 8 && warp < 12) {
        // ---- fetching
        const int ft = tid - 288;
        const long long bk = (long long)b * a.Hk + h / (a.H / a.Hk), qk = bk * a.Dk * a.L, all = (long long)a.B * a.Hk * a.Dk * a.L;
        for (int c = first, i = 0; c < last; ++c, ++i) {
            const int s = i % C::STAGES, t0 = c * kTok, nv = n - t0 < kTok ? n - t0 : kTok;
            unsigned char *st = sm + s * C::STAGE;
            const bool copied = by_copy(a, nv, t0), values = C::VALUES && !phi;
            if (copied && ft) continue;                      // (one thread's work)
            // one thread waits, for every chunk in turn: the others have passed over copied ones, and a barrier's parity tells them nothing
            if (i >= C::STAGES && ft == 0) WAIT(&ws.empty[s], (i / C::STAGES - 1) & 1);
            if (!copied) fetchers_sync();
            const bool begun = ft == 0 && !walk_given_up(&ws);
            if (begun) {
                const long long at = bh * a.chunks + c;
                ++ws.begun[s];
                const unsigned bytes = RUN ? C::IMAGES : C::PA * kMatrix, tiles = copied ? (RUN ? 2 : 1) * C::TENSOR + (values ? C::TILE : 0) : 0;
                mbar_expect_tx(&ws.full[s], bytes + kWalkGates + 16 + tiles);
                if (copied) {
                    tma_load_3d(st, &maps.k, &ws.full[s], t0, 0, (int)bk);
                    if (RUN) tma_load_3d(st + C::Q, &maps.q, &ws.full[s], t0, 0, (int)bk);
                    if (values) tma_load_3d(st + C::V, &maps.v, &ws.full[s], t0, 0, (int)bh);
                }
                bulk_load(st + C::A, a.images + at * C::IMAGES, bytes, &ws.full[s]);
                bulk_load(st + C::GATES, a.gates + at * kGates, kWalkGates, &ws.full[s]);
                bulk_load(&ws.carry[s], a.gates + at * kGates + kCarry, 16, &ws.full[s]);
            }
            if (!copied) {
                load_tile<T>(st, C::TILE, (const T *)a.k, qk + t0, all, a.L, a.Dk, nv, ft, kFetchers);
                if (RUN) load_tile<T>(st + C::Q, C::TILE, (const T *)a.q, qk + t0, all, a.L, a.Dk, nv, ft, kFetchers);
                if constexpr (C::VALUES)
                    if (values) load_tile<T>(st + C::V, C::TILE, (const T *)a.v, vhead + t0, vall, a.L, a.Dv, nv, ft, kFetchers);
                fence_async_smem();
                fetchers_sync();
            }
            if (begun) mbar_arrive(&ws.full[s]);
        }
    } else if (warp == 8) {
        // ---- the products
        const int steps = (a.Dk + 15) / 16;
        for (int c = first, i = 0; c < last; ++c, ++i) {
            const int s = i % C::STAGES;
            const unsigned par = i & 1, k = smem_u32(sm) + s * C::STAGE, A = k + C::A, P = A + C::PA * kMatrix;
            walk_late(&ws, is_late(a, KERNEL, bh, c, LATE_COPIES));
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            // S k, the first half of S's columns as soon as they are there
            WAIT(&ws.state[0], par);
            tmem_fence_after_sync();
            issue_ts<PM, PI, PM, true, KD / 32>(tb + C::X0, tb + C::S0, KD / 2, k, C::TILE, steps, kTok, false);
            WAIT(&ws.state[1], par);
            tmem_fence_after_sync();
            if (a.Dk > KD / 2) issue_ts<PM, PI, PM, true, KD / 32>(tb + C::X0, tb + C::S0 + KD / 4, KD / 2, k + KD / 2 * 128, C::TILE, steps - KD / 32, kTok, true);
            umma_commit(&ws.bar_a);
            if (RUN) {
                if (i) WAIT(&ws.o_taken, par ^ 1);           // (y of the chunk before)
                tmem_fence_after_sync();
                issue_ts<PM, PI, PM, true, KD / 16>(tb + C::Y0, tb + C::S0, KD / 2, k + C::Q, C::TILE, steps, kTok, false);
                umma_commit(&ws.bar_q);
            }
            WAIT(&ws.z_ready, par);
            tmem_fence_after_sync();
            issue_ts<PM, C::PA, C::PA, false, kTok / 16, B_LOWER>(tb + C::X0, tb + C::Z0, kTok / 2, A, kMatrix, kTok / 16, kTok, false);
            umma_commit(&ws.bar_b);
            WAIT(&ws.u_ready, par);
            tmem_fence_after_sync();
            issue_ts<PM, PI, PM, false, kTok / 16>(tb + C::D0, tb + C::U0, kTok / 2, k, C::TILE, kTok / 16, KD / 2, false);
            if (C::ROOM) umma_commit(&ws.bar_c[0]);
            issue_ts<PM, PI, PM, false, kTok / 16>(tb + C::D1, tb + C::U0, kTok / 2, k + KD / 2 * 128, C::TILE, kTok / 16, KD / 2, false);
            if (!C::ROOM) umma_commit(&ws.bar_c[0]);
            umma_commit(&ws.bar_c[1]);
            if (RUN) {
                WAIT(&ws.p_ready, par);
                WAIT(&ws.o_ready, par);                      // (y's first sum times gamma)
                tmem_fence_after_sync();
                issue_ts<PM, PM, PM, false, kTok / 16, B_LOWER>(tb + C::Y0, tb + C::Z0, kTok / 2, P, kMatrix, kTok / 16, kTok, true);
                umma_commit(&ws.bar_y);
            }
            umma_commit(&ws.empty[s]);
        }
        // (the last arrival on a barrier that nobody waits for comes before the CTA ends)
        if (last > first) WAIT(&ws.empty[(last - first - 1) % C::STAGES], ((last - first - 1) / C::STAGES) & 1);
    } else if (warp >= 12) {
        // ---- results: y's first sum times gamma, then y as an image that a copy takes away, or by these threads
        const int row = 32 * (warp & 3) + lane;
        const unsigned lane_y = tmem_addr(tb, warp, C::Y0);
        const long long vrow = vhead + (long long)row * a.L;
        const bool real = row < a.Dv, stored = C::VALUES && a.copies;
        for (int c = first, i = 0; RUN && c < last; ++c, ++i) {
            const int s = i % C::STAGES, t = c * kTok;
            const float *gates = (const float *)(sm + s * C::STAGE + C::GATES);
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            WAIT(&ws.bar_q, i & 1);
            tmem_fence_after_sync();
#pragma unroll 2
            for (int e = 0; e < kTok; e += 8) {
                f2 y[4], ga[4];
                tmem_ld8(y, lane_y + e);
                shared8(ga, gates + e);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = mul2(y[j], ga[j]);
                tmem_st8(lane_y + e, y);
            }
            walk_ready(&ws.o_ready, lane);
            unsigned char *image = sm + C::STAGES * C::STAGE + (i & 1) * C::TILE;
            walk_late(&ws, is_late(a, KERNEL, bh, c, LATE_RESULT));
            WAIT(&ws.bar_y, i & 1);
            tmem_fence_after_sync();
            auto put = [&](int e, const float (&y)[8]) {
                if (C::VALUES && stored) {
                    if (row < KD) *(uint4 *)(image + image_at(row, e >> 3)) = bf16_8(y, n - t - e);
                } else if (real && t + e < a.L) store8<T>((T *)a.y, vrow + t + e, a.L, a.L - t - e, n - t - e, y);
            };
#pragma unroll 2
            for (int e = 0; e < kTok; e += 8) {
                float y[8];
                tmem_ld8(y, lane_y + e);
                tmem_wait_ld();
                put(e, y);
            }
            walk_ready(&ws.o_taken, lane);
            if (walk_given_up(&ws)) {
                const float y[8] = {kLost, kLost, kLost, kLost, kLost, kLost, kLost, kLost};
#pragma unroll 1
                for (int e = 0; e < kTok; e += 8) put(e, y);
                __syncwarp();
            }
            if (stored) {
                fence_async_smem();
                takers_sync();
                if (tid == 384) {
                    tma_store_3d(&maps.out, image, t, 0, (int)bh);
                    tma_commit();
                    tma_wait_read1();                        // the other image is free again
                }
                takers_sync();
            }
        }
        if (RUN) {
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int t = kTok * (first > last ? first : last); t < kTok * end; t += 8)
                if (real && t < a.L) store8<T>((T *)a.y, vrow + t, a.L, a.L - t, 0, none);
            if (stored && tid == 384) tma_wait_all0();
        }
        tmem_fence_before_sync();
    } else {
        // ---- computing: lane of tensor memory = row of the state, `half` = which half of the columns
        const int row = 32 * (warp & 3) + lane, half = warp >> 2, rows = phi ? a.Dk : a.Dv;
        const unsigned lane_s = tmem_addr(tb, warp, C::S0 + half * (HC / 2)), lane_z = tmem_addr(tb, warp, C::Z0 + half * 16), lane_u = tmem_addr(tb, warp, C::U0 + half * 16),
                       lane_x = tmem_addr(tb, warp, C::X0 + half * 32), lane_d = tmem_addr(tb, warp, half ? C::D1 : C::D0);
        const bool values = row < a.Dv && !phi;
        f2 S[HC / 2];
        {
            float s[HC];
#pragma unroll
            for (int i = 0; i < HC; ++i) s[i] = phi && row == half * HC + i && row < a.Dk ? 1.f : 0.f;
            if (RUN && a.segments > 1) load_kept<HC>(s, a.starts + (bh * a.segments + segment) * kept_floats(a.Dv, a.Dk), row, a.Dv, half * HC, a.Dk);
            else if (RUN && a.s0) load_state<HC>(s, a.s0 + bh * states, row, a.Dv, half * HC, a.Dk);
#pragma unroll
            for (int i = 0; i < HC / 2; ++i) S[i] = make2(s[2 * i], s[2 * i + 1]);
        }
        planes_to_tmem<PM, HC / 2>(lane_s, KD / 2, S);
        for (int c = first, i = 0; c < last; ++c, ++i) {
            const int s = i % C::STAGES, t = c * kTok + 32 * half;
            const unsigned par = i & 1;
            const unsigned char *st = sm + s * C::STAGE;
            const float *gates = (const float *)(st + C::GATES) + 32 * half;
            walk_ready(&ws.state[half], lane);
            f2 held[C::VALUES ? 1 : 16];                     // (fp32 values come from device memory: ahead of their use)
            if constexpr (!C::VALUES) load_row(held, (const float *)a.v, vhead + (long long)row * a.L + t, a.L, values ? n - t : 0);
            float *mark = RUN && a.marks ? a.marks + (bh * a.chunks + c) * kept_floats(a.Dv, a.Dk) : nullptr;
            if (mark) keep_state<0, HC / 16>(mark, S, row, a.Dv, half * HC, a.Dk);
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            uint4 packed[C::VALUES ? 4 : 1];
            if constexpr (C::VALUES)
#pragma unroll
                for (int g = 0; g < 4; ++g) packed[g] = values ? *(const uint4 *)(st + C::V + image_at(row, 4 * half + g)) : make_uint4(0, 0, 0, 0);
            WAIT(&ws.bar_a, par);
            tmem_fence_after_sync();
            f2 x[16];
            tmem_ld(x, lane_x);
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < 4; ++g) {                    // Z = beta v - beta gamma S k
                f2 z[4], be[4], bg[4];
                if constexpr (C::VALUES) {
                    z[0] = widen2(packed[g].x); z[1] = widen2(packed[g].y); z[2] = widen2(packed[g].z); z[3] = widen2(packed[g].w);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = held[4 * g + e];
                }
                shared8(be, gates + 2 * kTok + 8 * g);
                shared8(bg, gates + 3 * kTok + 8 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = fma2(bg[e], x[4 * g + e], mul2(be[e], z[e]));
                planes8_to_tmem<PM>(lane_z + 4 * g, kTok / 2, z);
            }
            walk_ready(&ws.z_ready, lane);
            if (mark) keep_state<HC / 16, HC / 8>(mark, S, row, a.Dv, half * HC, a.Dk);
            const Carry carry(&ws.carry[s].x);
            walk_late(&ws, is_late(a, KERNEL, bh, c, LATE_PRODUCT));
            WAIT(&ws.bar_b, par);
            tmem_fence_after_sync();
            tmem_ld(x, lane_x);
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f2 u[4], de[4];
                shared8(de, gates + kTok + 8 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = mul2(x[4 * g + e], de[e]);
                planes8_to_tmem<PM>(lane_u + 4 * g, kTok / 2, u);
            }
            walk_ready(&ws.u_ready, lane);
            if (RUN) {
                planes_to_tmem<PM, 16>(lane_z, kTok / 2, x);
                walk_ready(&ws.p_ready, lane);
            }
            if (mark) keep_state<HC / 8, HC / 4>(mark, S, row, a.Dv, half * HC, a.Dk);
            WAIT(&ws.bar_c[half], par);
            tmem_fence_after_sync();
            state_onwards<PM>(S, carry, lane_d, lane_s, KD / 2);
            if (walk_given_up(&ws))
#pragma unroll
                for (int j = 0; j < HC / 2; ++j) S[j] = pair(kLost);
        }
        tmem_wait_st();
        auto flat = [&](float (&s)[HC]) {
#pragma unroll
            for (int i = 0; i < HC / 2; ++i) split2(S[i], s[2 * i], s[2 * i + 1]);
        };
        if (!RUN) {
            const int pitch = map_pitch(a.Dk);
            float *to = a.maps + ((bh * a.segments + segment) * (a.Dv + a.Dk) + (phi ? a.Dv : 0)) * (long long)pitch, s[HC];
            flat(s);
            store_state<HC>(to, s, row, rows, half * HC, pitch);
        } else {
            if (a.s_end && segment == a.segments - 1) {
                float s[HC];
                flat(s);
                store_state<HC>(a.s_end + bh * states, s, row, a.Dv, half * HC, a.Dk);
            }
        }
        tmem_fence_before_sync();
    }
    walk_end(&ws, C::STAGES, &hn_delta_status, warp, 8);
    if (warp == 0) tmem_dealloc(tb, 512);
    pdl_trigger();                                           // (late: see delta.cuh)
}

// ---- segments -------------------------------------------------------------------------------------------------------

// States at the segments' starts from the maps S -> S Phi + N: eight rows to a CTA, Phi by bulk copies, the next one under way; a thread
// sums four columns of all rows over an eighth of Phi's rows.  `reverse`: from the last segment to the first (the gradient's states).
// Serial over the segments: 37 of 128 channels take 56 us, 1.5 us each, for 64 KB that every CTA reads from L2 and 128 x 128 x 8 fp32 products.
constexpr int kJoinRows = 8, kJoinBytes = 2 * 128 * 128 * 4;
__global__ void __launch_bounds__(256) delta_join_kernel(DeltaArgs a, const float *from, int reverse)
{
    constexpr int R = kJoinRows;
    extern __shared__ __align__(16) float phi[];             // two of [Dk][pitch]
    __shared__ __align__(16) float S[R][128], part[8][R][128];
    __shared__ WalkShared ws;
    const int tid = threadIdx.x, quad = tid & 31, eighth = tid >> 5, tiles = (a.Dv + R - 1) / R, pitch = map_pitch(a.Dk), n = a.segments, step = reverse ? -1 : 1;
    const long long bh = blockIdx.x / tiles, states = (long long)a.Dv * a.Dk, map = (long long)(a.Dv + a.Dk) * pitch;
    const int row = (int)(blockIdx.x % tiles) * R + eighth, each = (a.Dk + 31) / 32 * 4;          // (a thread's row of S; Phi's rows of an eighth)
    const unsigned bytes = (unsigned)(a.Dk * pitch * 4);
    for (int e = tid; e < 2 * 128 * 128 / 4; e += 256) ((float4 *)phi)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tid == 0) {
        mbar_init(&ws.full[0], 1); mbar_init(&ws.full[1], 1);
        walk_marks_init(&ws);
    }
    fence_async_smem();
    pdl_join();
    __syncthreads();
    auto fetch = [&](int i) {                                // (one thread) the i-th segment's
        const int s = reverse ? n - 1 - i : i;
        ++ws.begun[i & 1];
        mbar_expect_tx(&ws.full[i & 1], bytes);
        bulk_load(phi + (i & 1) * 128 * 128, a.maps + (bh * n + s) * map + (long long)a.Dv * pitch, bytes, &ws.full[i & 1]);
    };
    if (tid == 0 && n > 1) fetch(0);
    if (tid == 0 && n > 2) fetch(1);
    // a warp holds a row: four columns a lane
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float *const mine = (float *)&v;
    if (from && row < a.Dv)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (4 * quad + e < a.Dk) { const float *p = from + bh * states + (long long)row * a.Dk + 4 * quad + e; HN_G(p, 4); mine[e] = *p; }
    for (int i = 0, s = reverse ? n - 1 : 0; i < n; ++i, s += step) {
        *(float4 *)&S[eighth][4 * quad] = v;
        if (row < kept_rows(a.Dv) && 4 * quad < a.Dk) {
            float4 *p = (float4 *)(a.starts + (bh * n + s) * kept_floats(a.Dv, a.Dk)) + kept_at(row, quad, kept_rows(a.Dv));
            HN_G(p, 16);
            *p = v;
        }
        if (i == n - 1) break;
        float4 add = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < a.Dv && 4 * quad < pitch) { const float4 *p = (const float4 *)(a.maps + (bh * n + s) * map + (long long)row * pitch) + quad; HN_G(p, 16); add = *p; }
        __syncthreads();
        walk_late(&ws, is_late(a, LATE_JOIN, bh, s, LATE_COPIES));
        WAIT(&ws.full[i & 1], (i >> 1) & 1);
        f2 acc[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][0] = acc[r][1] = pair(0.f);
        const float *w = phi + (i & 1) * 128 * 128 + eighth * each * pitch + 4 * quad;
        if (4 * quad < pitch)
            for (int k = 0; k < each; k += 4) {
                float4 p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = *(const float4 *)(w + (k + e) * pitch);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 q = *(const float4 *)&S[r][eighth * each + k];
                    const float qk[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[r][0] = fma2(pair(qk[e]), make2(p[e].x, p[e].y), acc[r][0]);
                        acc[r][1] = fma2(pair(qk[e]), make2(p[e].z, p[e].w), acc[r][1]);
                    }
                }
            }
#pragma unroll
        for (int r = 0; r < R; ++r) *(float4 *)&part[eighth][r][4 * quad] = make_float4(acc[r][0].x, acc[r][0].y, acc[r][1].x, acc[r][1].y);
        __syncthreads();
        if (tid == 0 && i + 2 < n - 1 && !walk_given_up(&ws)) fetch(i + 2);          // (every thread has read this one)
        v = add;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float4 p = *(const float4 *)&part[e][eighth][4 * quad];
            v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
        }
        if (walk_given_up(&ws)) v = make_float4(kLost, kLost, kLost, kLost);
    }
    walk_end(&ws, 2, &hn_delta_status, 0, -1);
}

// ---- one token ------------------------------------------------------------------------------------------------------

// W lanes to a row of the state, four columns each; the products with k and q are formed in one reading, the new state is written in
// the same: bandwidth is the bound (32 sequences of 6 heads of 128 channels: 25 MB of states in and out, 6.6 us; 3.9 at the rate of a
// copy).  A decay next to 1 is applied as a - 1, so that thousands of tokens one by one cost a rounding each.
template <typename T, int W> __global__ void __launch_bounds__(256) delta_step_kernel(DeltaArgs a)
{
    constexpr int ROWS = 256 / W, EACH = 4;                  // rows at a time, and times
    const int lane = threadIdx.x % W, c0 = 4 * lane, tiles = (a.Dv + ROWS * EACH - 1) / (ROWS * EACH);
    const long long bh = blockIdx.x / tiles;
    const int b = (int)(bh / a.H), h = (int)(bh % a.H), r0 = (int)(blockIdx.x % tiles) * ROWS * EACH + threadIdx.x / W;
    pdl_join();
    const float *from = a.s0 + bh * a.Dv * a.Dk;
    float *to = a.s_end + bh * a.Dv * a.Dk;
    float S[EACH][4], k[4], q[4];
#pragma unroll
    for (int e = 0; e < EACH; ++e) load_state<4>(S[e], from, r0 + e * ROWS, a.Dv, c0, a.Dk);
    bool in = true;
    if (a.lengths) { HN_G(a.lengths + b, 4); in = __ldg(a.lengths + b) > 0; }
    const long long qk = ((long long)b * a.Hk + h / (a.H / a.Hk)) * a.Dk, vr = bh * a.Dv;
    float kq = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k[i] = in && c0 + i < a.Dk ? IO<T>::ld((const T *)a.k, qk + c0 + i) : 0.f;
        q[i] = in && c0 + i < a.Dk ? IO<T>::ld((const T *)a.q, qk + c0 + i) : 0.f;
        kq = fmaf(k[i], q[i], kq);
    }
    float fade = 1.f, less = 0.f, beta = 0.f;
    if (in) {
        HN_G(a.beta + bh, 4);
        beta = __ldg(a.beta + bh);
        if (a.decay != DELTA_NONE) {
            HN_G(a.g + bh, 4);
            const float g = __ldg(a.g + bh);
            if (a.decay == DELTA_LOG) { fade = expf(g); less = expm1f(g); }
            else { const float e = expf(-fabsf(g)), x = e / (1.f + e); fade = g >= 0.f ? 1.f - x : x; less = g >= 0.f ? -x : x - 1.f; }
        }
    }
#pragma unroll
    for (int m = 1; m < W; m <<= 1) kq += __shfl_xor_sync(~0u, kq, m);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int r = r0 + e * ROWS;
        float sk = 0.f, sq = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) { sk = fmaf(S[e][i], k[i], sk); sq = fmaf(S[e][i], q[i], sq); }
#pragma unroll
        for (int m = 1; m < W; m <<= 1) { sk += __shfl_xor_sync(~0u, sk, m); sq += __shfl_xor_sync(~0u, sq, m); }
        float v = 0.f;
        if (in && r < a.Dv) v = IO<T>::ld((const T *)a.v, vr + r);
        const float u = beta * fmaf(-fade, sk, v);
        if (in) {
#pragma unroll
            for (int i = 0; i < 4; ++i) S[e][i] = fade > 0.5f ? S[e][i] + fmaf(less, S[e][i], u * k[i]) : fmaf(fade, S[e][i], u * k[i]);
        }
        if (r < a.Dv && lane == 0) IO<T>::st((T *)a.y, vr + r, in ? fmaf(fade, sq, u * kq) : 0.f);
        store_state<4>(to, S[e], r, a.Dv, c0, a.Dk);
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------

static size_t up(size_t n) { return (n + 255) / 256 * 256; }
DeltaSizes delta_sizes(const DeltaArgs &a, int dtype, bool backward)
{
    const size_t bh = (size_t)a.B * a.H, chunks = bh * a.chunks, planes = dtype == HYENAND_F32 ? Planes<float>::MID : Planes<bf16>::MID;
    DeltaSizes s{};
    s.images = chunks * (Planes<bf16>::INVERSE + planes) * kMatrix;
    s.gates = up(chunks * kGates * 4);
    if (a.segments > 1) {
        s.maps = up(bh * a.segments * ((size_t)a.Dv + a.Dk) * map_pitch(a.Dk) * 4);
        s.starts = up(bh * a.segments * (size_t)kept_floats(a.Dv, a.Dk) * 4);
    }
    if (backward) {
        s.dstates = up(chunks * (size_t)kept_floats(a.Dv, a.Dk) * 4);
        s.dz = chunks * (size_t)kept_rows(a.Dv) * kTok * 4;
    }
    s.all = s.images + s.gates + s.maps + s.starts + s.dstates + s.dz;
    return s;
}
static void place_workspace(DeltaArgs &a, const DeltaSizes &s, void *workspace)
{
    unsigned char *p = (unsigned char *)workspace;
    a.images = p; p += s.images;
    a.gates = (float *)p; p += s.gates;
    a.maps = (float *)p; p += s.maps;
    a.starts = (float *)p; p += s.starts;
    a.dstates = (float *)p; p += s.dstates;
    a.dz = (float *)p;
}

template <typename T> static int launch_prepare(DeltaArgs a, cudaStream_t st)
{
    const long long blocks = (long long)a.B * a.H * a.chunks;
    DeltaMaps m{};
    a.copies = delta_maps<T>(m, a, a.Dk <= 64 ? 64 : 128, a.v, nullptr, nullptr);
    return a.Dk <= 64 ? launch_delta<delta_prepare_kernel<T, 64>>(a, blocks, 128, Prep<T, 64>::BYTES, st, m)
                      : launch_delta<delta_prepare_kernel<T, 128>>(a, blocks, 128, Prep<T, 128>::BYTES, st, m);
}
int launch_delta_prepare(DeltaArgs a, int dtype, cudaStream_t st) { return dtype == HYENAND_F32 ? launch_prepare<float>(a, st) : launch_prepare<bf16>(a, st); }

int launch_delta_join(const DeltaArgs &a, const float *from, bool backward, cudaStream_t st)
{
    return launch_delta<delta_join_kernel>(a, (long long)a.B * a.H * ((a.Dv + kJoinRows - 1) / kJoinRows), 256, kJoinBytes, st, from, (int)backward);
}

template <typename T, int KD> static int launch_walk(DeltaArgs a, cudaStream_t st)
{
    DeltaMaps m{};
    a.copies = delta_maps<T>(m, a, KD, a.v, a.y, nullptr);
    const long long blocks = (long long)a.B * a.H * a.segments;
    if (a.segments > 1) {
        if (const int e = launch_delta<delta_walk_kernel<T, KD, WALK_MAPS>>(a, 2 * blocks, kWalkThreads, Walk<T, KD>::BYTES, st, m)) return e;
        if (const int e = launch_delta_join(a, a.s0, false, st)) return e;
    }
    return launch_delta<delta_walk_kernel<T, KD, WALK_RUN>>(a, blocks, kWalkThreads, Walk<T, KD>::BYTES, st, m);
}
template <typename T> static int launch_forward(const DeltaArgs &a, cudaStream_t st)
{
    if (const int e = launch_prepare<T>(a, st)) return e;
    return a.Dk <= 64 && a.Dv <= 64 ? launch_walk<T, 64>(a, st) : launch_walk<T, 128>(a, st);
}
template <typename T> static int launch_step(const DeltaArgs &a, cudaStream_t st)
{
    const int W = a.Dk <= 32 ? 8 : a.Dk <= 64 ? 16 : 32, per = 256 / W * 4;
    const long long blocks = (long long)a.B * a.H * ((a.Dv + per - 1) / per);
    return W == 8 ? launch_delta<delta_step_kernel<T, 8>>(a, blocks, 256, 0, st)
           : W == 16 ? launch_delta<delta_step_kernel<T, 16>>(a, blocks, 256, 0, st) : launch_delta<delta_step_kernel<T, 32>>(a, blocks, 256, 0, st);
}

// Segments of a head.  They cost three walks in place of one (two CTAs for the maps), so they pay where each SM would otherwise have a
// quarter of a head or less, and from some length on.  Scans with one walk and with segments, us: 37 heads of 128 channels (four segments)
// of 128 chunks 441 and 397, of 64 channels 408 and 324, fp32 2373 and 1472; 48 heads (three) 462 and 499, 434 and 412, 2448 and 1937; 60 (two)
// 497 and 647, 445 and 535, 2533 and 2731; 8 heads of 16 chunks 70 and 61, 55 and 45, 212 and 120, of 8 chunks 49 and 57, 38 and 42, 122 and 111.
// The worst of the rule: 37 heads of 16 chunks 78 and 110, 67 and 75, 300 and 233.  Training steps have the same borders.
static int segments_of(long long heads, int chunks)
{
    const long long n = kSms / heads;
    if (n < 4 || chunks < 16) return 1;
    const long long each = (chunks + n - 1) / n, most = each > 4 ? each : 4;
    return (int)((chunks + most - 1) / most);
}

#ifdef HYENAND_DEBUG
static std::atomic<int> late_kernel{-1}, late_chunk{-1}, late_wait{-1};
#endif

static int fill(DeltaArgs &a, int B, int H, int Hk, int L, int Dk, int Dv, int decay, int dtype)
{
    if (B < 1 || H < 1 || Hk < 1 || L < 1 || Dk < 1 || Dv < 1) return fail(HYENAND_ERR_INVALID_ARG, "B, H, Hk, L, Dk and Dv must be >= 1");
    if (decay != DELTA_LOG && decay != DELTA_SIGMOID && decay != DELTA_NONE) return fail(HYENAND_ERR_INVALID_ARG, "unknown decay %d", decay);
    if (dtype != HYENAND_F32 && dtype != HYENAND_BF16) return fail(HYENAND_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (H % Hk) return fail(HYENAND_ERR_INVALID_ARG, "H = %d is no multiple of Hk = %d", H, Hk);
    if (Dk > 128 || Dv > 128) return fail(HYENAND_ERR_UNSUPPORTED, "heads of up to 128 channels (Dk = %d, Dv = %d)", Dk, Dv);
    if (L > (1 << 30)) return fail(HYENAND_ERR_UNSUPPORTED, "L = %d is above 2^30", L);
    if ((long long)B * H > (1 << 24)) return fail(HYENAND_ERR_UNSUPPORTED, "B * H is above 2^24");
#ifdef HYENAND_DEBUG
    a.late_kernel = late_kernel; a.late_chunk = late_chunk; a.late_wait = late_wait;
#endif
    a.B = B; a.H = H; a.Hk = Hk; a.L = L; a.Dk = Dk; a.Dv = Dv; a.decay = decay;
    a.chunks = (L + kTok - 1) / kTok;
    if ((long long)B * H * a.chunks > 0x3fffffffll) return fail(HYENAND_ERR_UNSUPPORTED, "B * H * L is above 2^36");
    a.segments = segments_of((long long)B * H, a.chunks);
    a.per_segment = (a.chunks + a.segments - 1) / a.segments;
    return HYENAND_OK;
}
static size_t state_bytes(const DeltaArgs &a) { return (size_t)a.B * a.H * a.Dv * a.Dk * sizeof(float); }
static size_t mark_bytes(const DeltaArgs &a) { return (size_t)a.B * a.H * a.chunks * kept_floats(a.Dv, a.Dk) * sizeof(float); }
// what every call takes: q, k, v, g, beta (of T tokens)
static int inputs(CallTensors &c, const DeltaArgs &a, size_t T, int dtype)
{
    if (!a.q || !a.k || !a.v || !a.beta) return fail(HYENAND_ERR_INVALID_ARG, "q, k, v, beta must be non-NULL");
    if ((a.g != nullptr) != (a.decay != DELTA_NONE)) return fail(HYENAND_ERR_INVALID_ARG, "g is given exactly where there is a decay");
    const size_t es = elsize(dtype) * T * a.B, gb = (size_t)a.B * a.H * T * sizeof(float);
    c.in("q", a.q, es * a.Hk * a.Dk); c.in("k", a.k, es * a.Hk * a.Dk); c.in("v", a.v, es * a.H * a.Dv);
    c.in("g", a.g, gb, 4); c.in("beta", a.beta, gb, 4);
    c.in("lengths", a.lengths, (size_t)a.B * sizeof(int), 4);
    return HYENAND_OK;
}

}  // namespace hn

using namespace hn;

extern "C" long long hyenand_delta_marks(int L, int Dk, int Dv)
{
    return L < 1 || L > (1 << 30) || Dk < 1 || Dv < 1 || Dk > 128 || Dv > 128 ? 0 : (L + kTok - 1) / kTok * kept_floats(Dv, Dk);
}

extern "C" long long hyenand_delta_workspace_bytes(int B, int H, int Hk, int L, int Dk, int Dv, int dtype, int backward)
{
    clear_error();
    DeltaArgs a{};
    if (fill(a, B, H, Hk, L, Dk, Dv, DELTA_NONE, dtype)) return 0;
    return (long long)delta_sizes(a, dtype, backward != 0).all;
}

extern "C" int hyenand_debug_delta_late(int kernel, int chunk, int wait)
{
#ifdef HYENAND_DEBUG
    late_kernel = kernel; late_chunk = chunk; late_wait = wait;
    return 0;
#else
    (void)kernel; (void)chunk; (void)wait;
    return -1;
#endif
}

extern "C" int hyenand_delta_device_status(void)
{
    int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, hn_delta_status, sizeof(int)) != cudaSuccess) return -1;
    const int w = delta_backward_status();
    return w < 0 ? w : v | w;
}

extern "C" int hyenand_delta_forward(int B, int H, int Hk, int L, int Dk, int Dv, int decay, int dtype, const void *q, const void *k, const void *v,
                                     const float *g, const float *beta, const float *s0, const int *lengths, void *y, float *s_end, float *marks,
                                     void *workspace, void *cuda_stream)
{
    clear_error();
    DeltaArgs a{};
    if (int e = fill(a, B, H, Hk, L, Dk, Dv, decay, dtype)) return e;
    if (!y || !workspace) return fail(HYENAND_ERR_INVALID_ARG, "y and workspace must be non-NULL");
    a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.s0 = s0; a.lengths = lengths; a.y = y; a.s_end = s_end; a.marks = marks;
    CallTensors c;
    if (int e = inputs(c, a, L, dtype)) return e;
    const DeltaSizes s = delta_sizes(a, dtype, false);
    place_workspace(a, s, workspace);
    c.in("s0", s0, state_bytes(a));
    c.out("y", y, (size_t)B * H * Dv * L * elsize(dtype)); c.out("s_end", s_end, state_bytes(a), 16, "s0");
    c.out("marks", marks, mark_bytes(a)); c.out("workspace", workspace, s.all);
    if (int e = c.check()) return e;
    c.register_ranges();
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return finish(dtype == HYENAND_F32 ? launch_forward<float>(a, st) : launch_forward<bf16>(a, st));
}

extern "C" int hyenand_delta_backward(int B, int H, int Hk, int L, int Dk, int Dv, int decay, int dtype, const void *q, const void *k, const void *v,
                                      const float *g, const float *beta, const int *lengths, const float *marks, const void *dy, const float *ds_end,
                                      void *dq, void *dk, void *dv, float *dg, float *dbeta, float *ds0, void *workspace, void *cuda_stream)
{
    clear_error();
    DeltaArgs a{};
    if (int e = fill(a, B, H, Hk, L, Dk, Dv, decay, dtype)) return e;
    if (!marks || !dy || !dq || !dk || !dv || !dbeta || !workspace)
        return fail(HYENAND_ERR_INVALID_ARG, "marks, dy, dq, dk, dv, dbeta, workspace must be non-NULL");
    a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.lengths = lengths; a.marks = (float *)marks; a.dy = dy; a.ds_end = ds_end;
    a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.dbeta = dbeta; a.ds0 = ds0;
    CallTensors c;
    if (int e = inputs(c, a, L, dtype)) return e;
    if (decay == DELTA_NONE && dg) return fail(HYENAND_ERR_INVALID_ARG, "dg of a rule without a decay");
    const DeltaSizes s = delta_sizes(a, dtype, true);
    place_workspace(a, s, workspace);
    const size_t es = elsize(dtype) * (size_t)L * B, gb = (size_t)B * H * L * sizeof(float);
    c.in("marks", marks, mark_bytes(a)); c.in("dy", dy, es * H * Dv); c.in("ds_end", ds_end, state_bytes(a));
    c.out("dq", dq, es * Hk * Dk); c.out("dk", dk, es * Hk * Dk); c.out("dv", dv, es * H * Dv); c.out("dg", dg, gb, 4); c.out("dbeta", dbeta, gb, 4);
    c.out("ds0", ds0, state_bytes(a), 16, "ds_end"); c.out("workspace", workspace, s.all);
    if (int e = c.check()) return e;
    c.register_ranges();
    return finish(launch_delta_backward(a, dtype, (cudaStream_t)cuda_stream));
}

extern "C" int hyenand_delta_step(int B, int H, int Hk, int Dk, int Dv, int decay, int dtype, const void *q, const void *k, const void *v, const float *g,
                                  const float *beta, const float *state, const int *active, void *y, float *new_state, void *cuda_stream)
{
    clear_error();
    DeltaArgs a{};
    if (int e = fill(a, B, H, Hk, 1, Dk, Dv, decay, dtype)) return e;
    if (!state || !y || !new_state) return fail(HYENAND_ERR_INVALID_ARG, "state, y, new_state must be non-NULL");
    a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.s0 = state; a.lengths = active; a.y = y; a.s_end = new_state;
    CallTensors c;
    if (int e = inputs(c, a, 1, dtype)) return e;
    c.in("state", state, state_bytes(a));
    c.out("y", y, (size_t)B * H * Dv * elsize(dtype)); c.out("new_state", new_state, state_bytes(a), 16, "state");
    if (int e = c.check()) return e;
    c.register_ranges();
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return finish(dtype == HYENAND_F32 ? launch_step<float>(a, st) : launch_step<bf16>(a, st));
}
