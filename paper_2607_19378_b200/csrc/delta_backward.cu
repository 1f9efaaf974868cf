// The gated delta rule: gradients, in chunks (formulas and number formats in delta.cuh).
//
// prepare: as in the forward pass.
// walk: from the last chunk to the first, a CTA per head: the gradient of the state.  As in the forward walk its rows are the lanes of
//     tensor memory and every product takes the one before as its operand there: dS k, then A^T dU, then the new dS.  It writes dV, dZ
//     (as images, for bf16) and the gradient behind every chunk.  Few heads and many chunks go in segments as there (dS0 = dS1 Phi + N).
// gradients: a CTA an SM takes the chunks of the heads of queries and keys one after the other: from the state before the chunk (the forward's mark) and the gradient
//     behind it, U again, then dQ, dK, and the sums for beta and, over what crosses each token, for the decay.  Value heads that share queries and keys follow
//     one another in the CTA, so their sum has one order and needs no atomics.
#include "delta.cuh"

namespace hn {

static __device__ int hn_delta_backward_status;
#define WAIT(bar, parity) walk_wait(&ws, bar, parity)

// ---- walk -----------------------------------------------------------------------------------------------------------

template <typename T, int KD> struct WalkBack {
    static constexpr int PI = Planes<T>::IN, PM = Planes<T>::MID, PA = Planes<T>::INVERSE, TILE = KD * 128, TENSOR = PI * TILE;
    static constexpr bool VALUES = PI == 1;                                   // dV and dZ's two planes travel as images
    static constexpr int IMAGES = (PA + PM) * kMatrix, K = 0, Q = TENSOR, DY = 2 * TENSOR, A = 3 * TENSOR, GATES = A + IMAGES, STAGE = GATES + kWalkGates;
    static constexpr int OUT = VALUES ? 3 * TILE : 0;
    // (the product of dY and P takes 128 rows of dY's image: with 64 it reads on into the images that follow, for rows nothing looks at)
    static constexpr int STAGES = 3 * STAGE + OUT <= kWalkBytes ? 3 : 2 * STAGE + OUT <= kWalkBytes ? 2 : 1;
    static constexpr int BYTES = STAGES * STAGE + OUT;
    // tensor memory: dS as an operand | dU, later -beta gamma dZ, as an operand | dS k, then dZ | P^T dY | what dS gains | gamma dY as an operand
    static constexpr int SCOLS = PM * KD / 2, ZCOLS = PM * kTok / 2, S0 = 0, Z0 = SCOLS, X0 = Z0 + ZCOLS, Y0 = X0 + kTok;
    // (with three planes of 128 columns gamma dY takes dS's place, and the first half of the gain dZ's)
    static constexpr bool ROOM = Y0 + kTok + KD + ZCOLS <= 512;
    static constexpr int D0 = ROOM ? Y0 + kTok : X0, D1 = ROOM ? D0 + KD / 2 : Y0 + kTok, G0 = ROOM ? D0 + KD : S0;
    static_assert((ROOM || (D1 + KD / 2 <= 512 && KD / 2 == kTok)) && BYTES <= kWalkBytes, "tensor and shared memory");
};

// As the forward walk, bound by its chain: 262 us for 96 heads of 4096 tokens of 128 channels, 4.1 us a chunk.  dZ leaves as the two planes that
// the gradients take, by copies out of shared memory (where that took 252 us, stored from registers in that order, 16 bytes a line, 281; in fp32 252, but
// the gradients then paid 45 us for turning it).
template <typename T, int KD, int MODE> __global__ void __launch_bounds__(kWalkThreads, 1) delta_walk_back_kernel(DeltaArgs a, const __grid_constant__ DeltaMaps maps)
{
    using C = WalkBack<T, KD>;
    constexpr int PI = C::PI, PM = C::PM, HC = KD / 2;
    constexpr bool RUN = MODE == WALK_RUN;
    constexpr int KERNEL = RUN ? LATE_BACK : LATE_BACK_MAPS;
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ WalkShared ws;
    unsigned char *const sm = raw;
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp(tid >> 5);
    long long id = blockIdx.x;
    const bool phi = !RUN && (id & 1);                       // from the identity, without dY
    if (!RUN) id >>= 1;
    const long long bh = id / a.segments;
    const int segment = (int)(id % a.segments), b = (int)(bh / a.H), h = (int)(bh % a.H);
    pdl_wait();
    const int n = live_tokens(a, b), first = segment * a.per_segment, end = first + a.per_segment < a.chunks ? first + a.per_segment : a.chunks;
    int last = (n + kTok - 1) / kTok;                        // chunks last - 1 .. first hold tokens
    last = last < end ? last : end;
    const int count = last > first ? last - first : 0;
    if (warp == 0) tmem_alloc(smem_u32(&ws.slot), 512);
    if (tid == 0) {
        walk_init(&ws, C::STAGES);
        walk_late(&ws, smem_u32(raw) & 1023u);               // (images that start elsewhere would be read wrongly: see kWalkBytes)
    }
    for (int s = 0; s < C::STAGES; ++s) {
        clear_rows(sm + s * C::STAGE, C::TILE, 2 * PI, a.Dk, KD, tid, kWalkThreads);
        clear_rows(sm + s * C::STAGE + C::DY, C::TILE, PI, phi ? 0 : a.Dv, KD, tid, kWalkThreads);
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
        for (int i = 0; i < count; ++i) {
            const int c = last - 1 - i, s = i % C::STAGES, t0 = c * kTok, nv = n - t0 < kTok ? n - t0 : kTok;
            unsigned char *st = sm + s * C::STAGE;
            const bool copied = by_copy(a, nv, t0);
            if (copied && ft) continue;                      // (one thread's work)
            // one thread waits, for every chunk in turn: the others have passed over copied ones, and a barrier's parity tells them nothing
            if (i >= C::STAGES && ft == 0) WAIT(&ws.empty[s], (i / C::STAGES - 1) & 1);
            if (!copied) fetchers_sync();
            const bool begun = ft == 0 && !walk_given_up(&ws);
            if (begun) {
                const long long at = bh * a.chunks + c;
                ++ws.begun[s];
                mbar_expect_tx(&ws.full[s], C::IMAGES + kWalkGates + 16 + (copied ? (phi ? 2 : 3) * C::TENSOR : 0));
                if (copied) {
                    tma_load_3d(st, &maps.k, &ws.full[s], t0, 0, (int)bk);
                    tma_load_3d(st + C::Q, &maps.q, &ws.full[s], t0, 0, (int)bk);
                    if (!phi) tma_load_3d(st + C::DY, &maps.v, &ws.full[s], t0, 0, (int)bh);
                }
                bulk_load(st + C::A, a.images + at * C::IMAGES, C::IMAGES, &ws.full[s]);
                bulk_load(st + C::GATES, a.gates + at * kGates, kWalkGates, &ws.full[s]);
                bulk_load(&ws.carry[s], a.gates + at * kGates + kCarry, 16, &ws.full[s]);
            }
            if (!copied) {
                load_tile<T>(st, C::TILE, (const T *)a.k, qk + t0, all, a.L, a.Dk, nv, ft, kFetchers);
                load_tile<T>(st + C::Q, C::TILE, (const T *)a.q, qk + t0, all, a.L, a.Dk, nv, ft, kFetchers);
                if (!phi) load_tile<T>(st + C::DY, C::TILE, (const T *)a.dy, vhead + t0, vall, a.L, a.Dv, nv, ft, kFetchers);
                fence_async_smem();
                fetchers_sync();
            }
            if (begun) mbar_arrive(&ws.full[s]);
        }
    } else if (warp == 8) {
        // ---- the products
        const int steps = (a.Dk + 15) / 16;
        for (int i = 0; i < count; ++i) {
            const int s = i % C::STAGES;
            const unsigned par = i & 1, k = smem_u32(sm) + s * C::STAGE, q = k + C::Q, A = k + C::A, P = A + C::PA * kMatrix;
            // what half h of dS's columns gains from an operand in tensor memory and an image of Dk rows
            auto gain = [&](int h, unsigned from, unsigned image, bool add) {
                issue_ts<PM, PI, PM, false, kTok / 16>(tb + (h ? C::D1 : C::D0), from, kTok / 2, image + h * (KD / 2) * 128, C::TILE, kTok / 16, KD / 2, add);
            };
            walk_late(&ws, is_late(a, KERNEL, bh, last - 1 - i, LATE_COPIES));
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            // (P^T dY of the chunk before has been read: its dU was there; so has dZ)
            issue_ss<PI, PM, PM, false, true, kTok / 16, B_LOWER_T>(tb + C::Y0, k + C::DY, C::TILE, 0, P, kMatrix, kTok / 16, kTok, false);
            // dS k, the first half of dS's columns as soon as they are there
            WAIT(&ws.state[0], par);
            tmem_fence_after_sync();
            issue_ts<PM, PI, PM, true, KD / 32>(tb + C::X0, tb + C::S0, KD / 2, k, C::TILE, steps, kTok, false);
            WAIT(&ws.state[1], par);
            tmem_fence_after_sync();
            if (a.Dk > KD / 2) issue_ts<PM, PI, PM, true, KD / 32>(tb + C::X0, tb + C::S0 + KD / 4, KD / 2, k + KD / 2 * 128, C::TILE, steps - KD / 32, kTok, true);
            umma_commit(&ws.bar_a);
            if (C::ROOM) {                                   // gamma dY waits for nothing
                WAIT(&ws.o_ready, par);
                tmem_fence_after_sync();
                gain(0, tb + C::G0, q, false);
                gain(1, tb + C::G0, q, false);
            }
            WAIT(&ws.z_ready, par);                          // dU
            tmem_fence_after_sync();
            issue_ts<PM, C::PA, C::PA, true, kTok / 16, B_LOWER_T>(tb + C::X0, tb + C::Z0, kTok / 2, A, kMatrix, kTok / 16, kTok, false);
            umma_commit(&ws.bar_b);
            WAIT(&ws.u_ready, par);                          // -beta gamma dZ (without the room, gamma dY too)
            tmem_fence_after_sync();
            if (!C::ROOM) {
                WAIT(&ws.o_ready, par);
                if (RUN) WAIT(&ws.o_taken, par);             // (the gain comes where dZ is)
                tmem_fence_after_sync();
                gain(0, tb + C::G0, q, false);
                gain(1, tb + C::G0, q, false);
            }
            gain(0, tb + C::Z0, k, true);
            if (C::ROOM) umma_commit(&ws.bar_c[0]);
            gain(1, tb + C::Z0, k, true);
            if (!C::ROOM) umma_commit(&ws.bar_c[0]);
            umma_commit(&ws.bar_c[1]);
            if (RUN && C::ROOM) WAIT(&ws.o_taken, par);      // (the gates are read there too)
            umma_commit(&ws.empty[s]);
        }
        // (the last arrival on a barrier that nobody waits for comes before the CTA ends)
        if (count) WAIT(&ws.empty[(count - 1) % C::STAGES], ((count - 1) / C::STAGES) & 1);
    } else if (warp >= 12) {
        // ---- gamma dY as an operand; dZ and dV on their way out
        const int row = 32 * (warp & 3) + lane, rows8 = kept_rows(a.Dv);
        const unsigned lane_g = tmem_addr(tb, warp, C::G0), lane_x = tmem_addr(tb, warp, C::X0);
        const long long vrow = vhead + (long long)row * a.L;
        const bool real = row < a.Dv, stored = C::VALUES && a.copies;
        for (int i = 0; i < count; ++i) {
            const int c = last - 1 - i, s = i % C::STAGES, t = c * kTok;
            const unsigned char *st = sm + s * C::STAGE;
            const float *gates = (const float *)(st + C::GATES);
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            WAIT(C::ROOM ? &ws.state[0] : &ws.bar_a, i & 1);          // its place is free: the gain before has been formed; or dS k has
            tmem_fence_after_sync();
#pragma unroll 2
            for (int e = 0; e < kTok; e += 8) {
                f2 x[4], ga[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = pair(0.f);
                if (real && !phi) {
                    float y[8];
                    image8<PI>(y, st + C::DY, C::TILE, row, e >> 3);
                    shared8(ga, gates + e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = mul2(make2(y[2 * j], y[2 * j + 1]), ga[j]);
                }
                __syncwarp();
                planes8_to_tmem<PM>(lane_g + e / 2, kTok / 2, x);
            }
            walk_ready(&ws.o_ready, lane);
            if (!RUN) continue;
            unsigned char *image = sm + C::STAGES * C::STAGE;
            if (C::VALUES) {
                if (tid == 384) tma_wait_read0();            // the images of the chunk before have been read
                __syncwarp();
                takers_sync();
            }
            walk_late(&ws, is_late(a, KERNEL, bh, c, LATE_RESULT));
            WAIT(&ws.bar_b, i & 1);
            tmem_fence_after_sync();
            float4 *to = (float4 *)a.dz + (bh * a.chunks + c) * 16 * rows8;     // dZ: two planes as images, or [quartet of tokens][row]
            auto put = [&](int e, const f2 (&z)[4], const f2 (&be)[4]) {
                if constexpr (C::VALUES) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) split2(z[j], x[2 * j], x[2 * j + 1]);
                    if (row < KD) planes8_to_image<PM>(image + C::TILE, C::TILE, row, e >> 3, x);
                } else if (row < rows8) {
                    float4 *at = to + (e >> 2) * rows8 + row;
                    HN_G(at, 16); HN_G(at + rows8, 16);
                    at[0] = make_float4(z[0].x, z[0].y, z[1].x, z[1].y);
                    at[rows8] = make_float4(z[2].x, z[2].y, z[3].x, z[3].y);
                }
                float y[8];                                  // dV: as an image that a copy takes away, or by these threads
#pragma unroll
                for (int j = 0; j < 4; ++j) split2(mul2(z[j], be[j]), y[2 * j], y[2 * j + 1]);
                if (C::VALUES && stored) {
                    if (row < KD) *(uint4 *)(image + image_at(row, e >> 3)) = bf16_8(y, n - t - e);
                } else if (real && t + e < a.L) store8<T>((T *)a.dv, vrow + t + e, a.L, a.L - t - e, n - t - e, y);
                __syncwarp();
            };
#pragma unroll 2
            for (int e = 0; e < kTok; e += 8) {
                f2 z[4], be[4];
                tmem_ld8(z, lane_x + e);
                shared8(be, gates + 2 * kTok + e);
                tmem_wait_ld();
                put(e, z, be);
            }
            walk_ready(&ws.o_taken, lane);                   // (the gates have been read as well)
            if (walk_given_up(&ws)) {
                const f2 z[4] = {pair(kLost), pair(kLost), pair(kLost), pair(kLost)};
#pragma unroll 1
                for (int e = 0; e < kTok; e += 8) put(e, z, z);
            }
            if (C::VALUES) {
                fence_async_smem();
                takers_sync();
                if (tid == 384) {
                    if (stored) tma_store_3d(&maps.out, image, t, 0, (int)bh);
                    for (int p = 0; p < 2; ++p) {
                        HN_G((unsigned char *)to + p * rows8 * 128, rows8 * 128);
                        bulk_store((unsigned char *)to + p * rows8 * 128, image + (p + 1) * C::TILE, rows8 * 128);
                    }
                    tma_commit();
                }
                __syncwarp();
            }
        }
        if (RUN) {
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int t = kTok * (first > last ? first : last); t < kTok * end; t += 8)
                if (real && t < a.L) store8<T>((T *)a.dv, vrow + t, a.L, a.L - t, 0, none);
            if (C::VALUES && tid == 384) tma_wait_all0();
        }
        tmem_fence_before_sync();
    } else {
        // ---- computing
        const int row = 32 * (warp & 3) + lane, half = warp >> 2, rows = phi ? a.Dk : a.Dv;
        const unsigned lane_s = tmem_addr(tb, warp, C::S0 + half * (HC / 2)),
                       lane_z = tmem_addr(tb, warp, C::Z0 + half * 16), lane_x = tmem_addr(tb, warp, C::X0 + half * 32), lane_y = tmem_addr(tb, warp, C::Y0 + half * 32),
                       lane_d = tmem_addr(tb, warp, half ? C::D1 : C::D0);
        f2 S[HC / 2];
        {
            float s[HC];
#pragma unroll
            for (int i = 0; i < HC; ++i) s[i] = phi && row == half * HC + i && row < a.Dk ? 1.f : 0.f;
            if (RUN && a.segments > 1) load_kept<HC>(s, a.starts + (bh * a.segments + segment) * kept_floats(a.Dv, a.Dk), row, a.Dv, half * HC, a.Dk);
            else if (RUN && a.ds_end) load_state<HC>(s, a.ds_end + bh * states, row, a.Dv, half * HC, a.Dk);
#pragma unroll
            for (int i = 0; i < HC / 2; ++i) S[i] = make2(s[2 * i], s[2 * i + 1]);
        }
        planes_to_tmem<PM, HC / 2>(lane_s, KD / 2, S);
        for (int i = 0; i < count; ++i) {
            const int c = last - 1 - i, s = i % C::STAGES;
            const unsigned par = i & 1;
            const float *gates = (const float *)(sm + s * C::STAGE + C::GATES) + 32 * half;
            walk_ready(&ws.state[half], lane);
            float *keep = RUN ? a.dstates + (bh * a.chunks + c) * kept_floats(a.Dv, a.Dk) : nullptr;
            if (RUN) keep_state<0, HC / 16>(keep, S, row, a.Dv, half * HC, a.Dk);
            WAIT(&ws.full[s], (i / C::STAGES) & 1);
            WAIT(&ws.bar_a, par);
            tmem_fence_after_sync();
            f2 x[16];
            tmem_ld(x, lane_x);
            Sixteen y[2];
            y[0].load(lane_y);
#pragma unroll
            for (int b = 0; b < 2; ++b) {                    // dU = P^T dY + delta dS k
                tmem_wait_ld();
                if (b == 0) y[1].load(lane_y + 16);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    f2 u[4], de[4];
                    shared8(de, gates + kTok + 16 * b + 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] = row < rows ? fma2(de[e], x[8 * b + 4 * g + e], phi ? pair(0.f) : y[b].get(4 * g + e)) : pair(0.f);
                    planes8_to_tmem<PM>(lane_z + 8 * b + 4 * g, kTok / 2, u);
                }
            }
            walk_ready(&ws.z_ready, lane);
            if (RUN) keep_state<HC / 16, HC / 8>(keep, S, row, a.Dv, half * HC, a.Dk);
            const Carry carry(&ws.carry[s].x);
            walk_late(&ws, is_late(a, KERNEL, bh, c, LATE_PRODUCT));
            WAIT(&ws.bar_b, par);
            tmem_fence_after_sync();
            tmem_ld(x, lane_x);
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f2 z[4], bg[4];
                shared8(bg, gates + 3 * kTok + 8 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = mul2(x[4 * g + e], bg[e]);
                planes8_to_tmem<PM>(lane_z + 4 * g, kTok / 2, z);
            }
            walk_ready(&ws.u_ready, lane);
            if (RUN) keep_state<HC / 8, HC / 4>(keep, S, row, a.Dv, half * HC, a.Dk);
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
            if (a.ds0 && segment == 0) {
                float s[HC];
                flat(s);
                store_state<HC>(a.ds0 + bh * states, s, row, a.Dv, half * HC, a.Dk);
            }
        }
        tmem_fence_before_sync();
    }
    walk_end(&ws, C::STAGES, &hn_delta_backward_status, warp, 8);
    if (warp == 0) tmem_dealloc(tb, 512);
    pdl_trigger();                                           // (late: see delta.cuh)
}

// ---- gradients ------------------------------------------------------------------------------------------------------

template <typename T, int KD> struct Grads {
    static constexpr int PI = Planes<T>::IN, PM = Planes<T>::MID, PA = Planes<T>::INVERSE, TILE = KD * 128;
    // images: dY | Q | K | U (values before it, dK in its second half behind it) | dZ (later E) | A (later F) | dQ, and a state as it is kept.
    // With three planes there is no room for the last two, and Q comes into dY's place once that is through.
    static constexpr bool ROOM = PI == 1;
    static constexpr int DY = 0, K = (ROOM ? 2 : 1) * PI * TILE, Q = ROOM ? PI * TILE : DY, U = (ROOM ? 3 : 2) * PI * TILE, DZ = U + PM * TILE, A = DZ + PM * TILE, OUT = A + PA * kMatrix,
                         STATE = OUT + (ROOM ? TILE : 0), BYTES = 1024 + STATE + (ROOM ? KD * KD * 4 : 0);
    // tensor memory: a state as an operand | sums of 64 columns:
    //     0: S0 k, U, the rest of dZ U^T   1: Z (and the next), dY U^T and dZ U^T   2: Q K^T and K K^T, the written part of dK but for dS1 u
    //     3: S0 dZ, the erased part of dK   4: S0 dY, dQ   5 (0 where there is no rest): dS1 u
    static constexpr bool REST = PI < PM;
    static constexpr int S0 = 0, SCOLS = PM * KD / 2, R0 = SCOLS, R1 = R0 + kTok, R2 = R1 + kTok, R3 = R2 + kTok, R4 = R3 + kTok, R5 = REST ? R4 + kTok : R0;
    static_assert(R4 + kTok <= 512 && R5 + kTok <= 512 && BYTES + 9728 <= 227 * 1024 && PM * kTok / 2 <= 2 * kTok && PM * TILE >= PM * kMatrix, "tensor and shared memory");
};
constexpr int kGradThreads = 512;

// x[c] summed over the warp's lanes: lanes 4 c .. 4 c + 3 are left with column c
__device__ __forceinline__ float column_sum8(float (&x)[8], int lane)
{
#pragma unroll
    for (int m = 4; m; m >>= 1) {
        const bool up = lane & (4 * m);
#pragma unroll
        for (int c = 0; c < m; ++c) {
            const float give = up ? x[c] : x[c + m], keep = up ? x[c + m] : x[c];
            x[c] = keep + __shfl_xor_sync(~0u, give, 4 * m);
        }
    }
    x[0] += __shfl_xor_sync(~0u, x[0], 1);
    return x[0] + __shfl_xor_sync(~0u, x[0], 2);
}

// 512 threads: a lane's columns in four quarters of 16 tokens (KD / 4 of a state), taken eight at a time: the loops stay rolled, as code that
// runs once per CTA is bound by its fetching (unrolled over 32 columns, 256 threads: 1350 us on 6144 chunks of 128 channels).
// 563 us on those, 13.6 us a chunk: 1.76 GB, of which the kept states and gradients in fp32 are 0.8, so 3.1 TB/s, and some 160 products of 34
// cycles, a fifth of the time.  What is left is the order of its six steps, each a write, a barrier, products, a reading.  The next chunk's
// copies go out as soon as their places are free (588 -> 525).  A warp of its own for the products made it slower (645 us: 17 warps leave a
// thread 96 registers, and the others run apart, through more code at a time).
template <typename T, int KD> __global__ void __launch_bounds__(kGradThreads, 1) delta_gradients_kernel(DeltaArgs a, const __grid_constant__ DeltaMaps maps)
{
    using C = Grads<T, KD>;
    constexpr int PI = C::PI, PM = C::PM, HC = KD / 4;
    extern __shared__ __align__(1024) unsigned char raw[];
    // bar_a, bar_b: products; full[0]: a unit's k, q, v, A, gates; full[1]: the gradient behind the chunk; full[2]: dY, the state before it
    __shared__ WalkShared ws;
    __shared__ __align__(16) float gates2[2][kGates];
    // sums over lanes, by the four warps of a quarter: dZ R | S0's part of a token's query and key | delta (dS1 u) k | a column's pairs in front
    // of it; a row's pairs in a quarter (rows 0 .. 63 of F, 64 .. of E without beta)
    __shared__ float sums[4][4][kTok], pairs[4][2 * kTok], total[16];
    unsigned char *sm = align_images(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform_warp(tid >> 5), row = 32 * (warp & 3) + lane, quarter = warp >> 2, share = a.H / a.Hk, c0 = 16 * quarter;
    const int rows8 = kept_rows(a.Dv), ksteps = (a.Dk + 15) / 16, vsteps = (a.Dv + 15) / 16;
    const long long all = (long long)a.B * a.Hk * a.Dk * a.L, vall = (long long)a.B * a.H * a.Dv * a.L, kept = kept_floats(a.Dv, a.Dk);
    const unsigned images = smem_u32(sm), IK = images + C::K, IU = images + C::U, IZ = images + C::DZ, IA = images + C::A, IY = images + C::DY, IQ = images + C::Q;
    // a unit: a chunk of a head of queries and keys, and one of the value heads that share it
    struct Unit { long long bk; int chunk, b, j, n, nv; };
    const long long items = (long long)a.B * a.Hk * a.chunks;
    auto unit = [&](long long item, int j) {
        Unit u;
        u.bk = item / a.chunks; u.chunk = (int)(item % a.chunks); u.b = (int)(u.bk / a.Hk); u.j = j;
        u.n = live_tokens(a, u.b);
        u.nv = u.n - u.chunk * kTok < kTok ? u.n - u.chunk * kTok : kTok;
        return u;
    };
    auto head = [&](const Unit &u) { return (long long)u.b * a.H + (u.bk % a.Hk) * share + u.j; };
    // the copies of a unit, in two parts: what can come while the unit before is still at its products, and the rest
    auto copy_early = [&](const Unit &u) {
        const long long bh = head(u), at = bh * a.chunks + u.chunk;
        const bool copied = by_copy(a, u.nv, u.chunk * kTok);
        ++ws.begun[2];
        mbar_expect_tx(&ws.full[2], (C::ROOM ? (unsigned)(kept * 4) : 0) + (copied ? C::TILE : 0));
        if (copied) tma_load_3d(sm + C::DY, &maps.v, &ws.full[2], u.chunk * kTok, 0, (int)bh);
        if (C::ROOM) bulk_load(sm + C::STATE, a.marks + at * kept, (unsigned)(kept * 4), &ws.full[2]);
    };
    auto copy_rest = [&](const Unit &u, int which) {
        const long long bh = head(u), at = bh * a.chunks + u.chunk;
        const bool copied = by_copy(a, u.nv, u.chunk * kTok);
        ++ws.begun[0];
        mbar_expect_tx(&ws.full[0], C::PA * kMatrix + kGates * 4 + (C::ROOM ? rows8 * 256 : 0) + (copied ? (u.j ? 1 : 3) * C::TILE : 0));
        if (copied) {
            if (!u.j) tma_load_3d(sm + C::K, &maps.k, &ws.full[0], u.chunk * kTok, 0, (int)u.bk);
            tma_load_3d(sm + C::U, &maps.more, &ws.full[0], u.chunk * kTok, 0, (int)bh);
            if (!u.j) tma_load_3d(sm + C::Q, &maps.q, &ws.full[0], u.chunk * kTok, 0, (int)u.bk);
        }
        bulk_load(gates2[which], a.gates + at * kGates, kGates * 4, &ws.full[0]);
        bulk_load(sm + C::A, a.images + at * ((C::PA + PM) * kMatrix), C::PA * kMatrix, &ws.full[0]);
        if (C::ROOM)
            for (int p = 0; p < 2; ++p) bulk_load(sm + C::DZ + p * C::TILE, (const unsigned char *)a.dz + (at * 2 + p) * rows8 * 128, rows8 * 128, &ws.full[0]);
    };
    pdl_wait();
    if (tid == 0) {
        mbar_init(&ws.bar_a, 1); mbar_init(&ws.bar_b, 1); mbar_init(&ws.full[0], 1); mbar_init(&ws.full[1], 1); mbar_init(&ws.full[2], 1);
        walk_marks_init(&ws);
    }
    __syncwarp();
    if (warp == 0) tmem_alloc(smem_u32(&ws.slot), 512);
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const unsigned tb = ws.slot;
    const unsigned lane_s = tmem_addr(tb, warp, C::S0 + quarter * (HC / 2)), lane_r = tmem_addr(tb, warp, c0);
    unsigned par = 0;
    float dq[2][8], dk[2][8];
    auto go = [&] {                                          // what the threads wrote, for the products
        tmem_wait_st();
        fence_async_smem();
        tmem_fence_before_sync();
        __syncthreads();
        tmem_fence_after_sync();
    };
    auto done = [&] {
        WAIT(&ws.bar_a, par);
        par ^= 1;
        tmem_fence_after_sync();
    };
    // the units of this CTA that hold tokens, one after the other; chunks without any are zeroed as they come
    long long item = (long long)blockIdx.x - gridDim.x;
    int j = share - 1;
    auto next = [&](Unit &u) {
        for (;;) {
            if (++j >= share) {
                j = 0;
                item += gridDim.x;
                if (item >= items) return false;
            }
            u = unit(item, j);
            if (u.nv > 0) return true;
            const int t = u.chunk * kTok, room = a.L - t < kTok ? a.L - t : kTok;
            const long long qrow = (u.bk * a.Dk + row) * a.L + t + c0;
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int g = 0; g < 16; g += 8)
                if (row < a.Dk && c0 + g < room) {
                    store8<T>((T *)a.dq, qrow + g, a.L, room - c0 - g, 0, none);
                    store8<T>((T *)a.dk, qrow + g, a.L, room - c0 - g, 0, none);
                }
            for (int i = tid; i < share * room; i += kGradThreads) {
                const long long at = (((long long)u.b * a.H + (u.bk % a.Hk) * share + i / room) * a.L) + t + i % room;
                HN_G(a.dbeta + at, 4);
                a.dbeta[at] = 0.f;
                if (a.dg) { HN_G(a.dg + at, 4); a.dg[at] = 0.f; }
            }
            j = share - 1;                                   // (the other heads of the chunk are done with)
        }
    };
    Unit now, then;
    bool more = next(now);
    if (more && tid == 0) { copy_early(now); copy_rest(now, 0); }
    __syncwarp();
    for (unsigned step = 0; more; ++step, now = then) {
        const unsigned phase = step & 1;
        const int t0 = now.chunk * kTok, nv = now.nv, room = a.L - t0 < kTok ? a.L - t0 : kTok, t = t0 + c0;
        const long long bh = head(now), at = bh * a.chunks + now.chunk, grow = bh * a.L + t0, qk = now.bk * a.Dk * a.L + t0;
        const float *S = a.marks + at * kept, *D = a.dstates + at * kept;
        const float *gates = gates2[phase], *gamma = gates, *delta = gates + kTok, *beta = gates + 2 * kTok, *ghi = gates + kSums, *glo = ghi + kTok;
        const bool copied = by_copy(a, nv, t0), first = now.j == 0, last = now.j == share - 1;
        more = next(then);
        if (first) {
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) dq[g][e] = dk[g][e] = 0.f;
        }
        if (!copied) {
            __syncthreads();                                 // (the results of the unit before have left U's place: their thread has waited)
            load_tile<T>(sm + C::DY, C::TILE, (const T *)a.dy, bh * a.Dv * a.L + t0, vall, a.L, a.Dv, nv, tid, kGradThreads);
            clear_rows(sm + C::DY, C::TILE, PI, a.Dv, KD, tid, kGradThreads);
            if (first) {
                load_tile<T>(sm + C::K, C::TILE, (const T *)a.k, qk, all, a.L, a.Dk, nv, tid, kGradThreads);
                clear_rows(sm + C::K, C::TILE, PI, a.Dk, KD, tid, kGradThreads);
                if (C::ROOM) {
                    load_tile<T>(sm + C::Q, C::TILE, (const T *)a.q, qk, all, a.L, a.Dk, nv, tid, kGradThreads);
                    clear_rows(sm + C::Q, C::TILE, PI, a.Dk, KD, tid, kGradThreads);
                }
            }
            load_tile<T>(sm + C::U, C::TILE, (const T *)a.v, bh * a.Dv * a.L + t0, vall, a.L, a.Dv, nv, tid, kGradThreads);
        }
        if (!C::ROOM) {                                      // dZ as an image
            const float4 *from = (const float4 *)a.dz + (at * 16 + 4 * quarter) * rows8 + row;
            float4 w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (row < rows8) { HN_G(from + e * rows8, 16); w[e] = from[e * rows8]; }
            }
            if (row < KD)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float x[8] = {w[2 * g].x, w[2 * g].y, w[2 * g].z, w[2 * g].w, w[2 * g + 1].x, w[2 * g + 1].y, w[2 * g + 1].z, w[2 * g + 1].w};
                    planes8_to_image<PM>(sm + C::DZ, C::TILE, row, 2 * quarter + g, x);
                }
        }
        WAIT(&ws.full[2], phase);
        const float4 *held = C::ROOM ? (const float4 *)(sm + C::STATE) : nullptr;
        // the state before the chunk, its rows as lanes: S0 k
#pragma unroll 1
        for (int e = 0; e < HC; e += 8) {
            float s[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const int c = quarter * HC + e + i;
                float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
                if (row < rows8 && c < a.Dk) {
                    const int k = kept_at(row, c >> 2, rows8);
                    if (C::ROOM) w = held[k];
                    else { HN_G((const float4 *)S + k, 16); w = ((const float4 *)S)[k]; }
                }
                s[i] = w.x; s[i + 1] = w.y; s[i + 2] = w.z; s[i + 3] = w.w;
            }
            planes8_to_tmem<PM>(lane_s + e / 2, KD / 2, s);
        }
        walk_late(&ws, is_late(a, LATE_GRADIENTS, bh, now.chunk, LATE_COPIES));
        WAIT(&ws.full[0], phase);
        if (C::ROOM) clear_rows(sm + C::DZ, C::TILE, PM, rows8, KD, tid, kGradThreads);
        go();
        if (warp == 0) {
            issue_ts<PM, PI, PM, true, KD / 16, B_ALL, 4>(tb + C::R0, tb + C::S0, KD / 2, IK, C::TILE, ksteps, kTok, false);
            umma_commit(&ws.bar_a);
            // rows 0 .. 63: Q K^T, rows 64 ..: K K^T
            if (C::ROOM) issue_ss<PI, PI, PI, true, true, KD / 16, B_ALL, 4>(tb + C::R2, IQ, C::TILE, C::K - C::Q, IK, C::TILE, ksteps, kTok, false);
        }
        done();
#pragma unroll 1
        for (int g = 0; g < 2; ++g) {                        // R, Z and what dZ R says about beta
            const int c = c0 + 8 * g;
            f2 x[4], ga[4], be[4];
            float v[8], z[8];
            tmem_ld8(x, lane_r + C::R0 + 8 * g);
            shared8(ga, gamma + c);
            shared8(be, beta + c);
            if (row < KD) {
                image8<PI>(v, sm + C::U, C::TILE, row, c >> 3);
                image8<PM>(z, sm + C::DZ, C::TILE, row, c >> 3);
            }
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = row < a.Dv ? fma2(mul2(ga[e], pair(-1.f)), x[e], make2(v[2 * e], v[2 * e + 1])) : pair(0.f);
                const f2 zr = mul2(make2(z[2 * e], z[2 * e + 1]), x[e]);
                z[2 * e] = row < a.Dv ? zr.x : 0.f;
                z[2 * e + 1] = row < a.Dv ? zr.y : 0.f;
                x[e] = mul2(x[e], be[e]);
            }
            planes8_to_tmem<PM>(tmem_addr(tb, warp, C::R1 + quarter * 8 + 4 * g), kTok / 2, x);
            const float sum = column_sum8(z, lane);
            if (!(lane & 3)) sums[0][warp & 3][c + (lane >> 2)] = sum;
        }
        go();
        if (warp == 0) {
            issue_ts<PM, C::PA, C::PA, false, kTok / 16, B_LOWER>(tb + C::R0, tb + C::R1, kTok / 2, IA, kMatrix, kTok / 16, kTok, false);
            umma_commit(&ws.bar_a);
        }
        // a state with its columns as lanes; `with`: the sum of its products with the one that is there
        auto columns = [&](const float *p, bool with) {
            float inner = 0.f;
            const int q7 = (row >> 2) & 7;
            const float *mine = (C::ROOM ? (const float *)held : p) + (row < a.Dk ? (row >> 2) * rows8 * 4 + (row & 3) : 0);
#pragma unroll 1
            for (int c = 0; c < HC; c += 8) {
                const int r = quarter * HC + c;              // rows r .. r + 7, all kept or none
                float s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = 0.f;
                if (r < rows8 && row < a.Dk) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (!C::ROOM) HN_G(mine + r * 4 + (e ^ q7) * 4, 4);
                        s[e] = mine[r * 4 + (e ^ q7) * 4];
                    }
                }
                __syncwarp();
                if (with) {
                    unsigned o[PM][4];
#pragma unroll
                    for (int q = 0; q < PM; ++q)
                        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];\n"
                                     : "=r"(o[q][0]), "=r"(o[q][1]), "=r"(o[q][2]), "=r"(o[q][3]) : "r"(lane_s + q * (KD / 2) + c / 2) : "memory");
                    tmem_wait_ld();
#pragma unroll
                    for (int q = 0; q < PM; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            inner = fmaf(__uint_as_float(o[q][e] << 16), s[2 * e], inner);
                            inner = fmaf(__uint_as_float(o[q][e] & 0xffff0000u), s[2 * e + 1], inner);
                        }
                }
                planes8_to_tmem<PM>(lane_s + c / 2, KD / 2, s);
            }
            return inner;
        };
        columns(S, false);
        go();
        if (warp == 0) {
            if (C::ROOM && lane == 0 && !walk_given_up(&ws)) {          // the state has been read: the gradient behind the chunk into its place
                ++ws.begun[1];
                mbar_expect_tx(&ws.full[1], (unsigned)(kept * 4));
                bulk_load(sm + C::STATE, D, (unsigned)(kept * 4), &ws.full[1]);
            }
            __syncwarp();
            issue_ts<PM, PI, PM, true, KD / 16, B_ALL, 4>(tb + C::R4, tb + C::S0, KD / 2, IY, C::TILE, vsteps, kTok, false);            // S0 dY
            issue_ts<PM, PM, PM, true, KD / 16, B_ALL, 4>(tb + C::R3, tb + C::S0, KD / 2, IZ, C::TILE, vsteps, kTok, false);            // S0 dZ
            umma_commit(&ws.bar_b);
        }
        done();
#pragma unroll 1
        for (int g = 0; g < 2; ++g) {
            float x[8];
            tmem_ld8(x, lane_r + C::R0 + 8 * g);
            tmem_wait_ld();
            if (row < KD) planes8_to_image<PM>(sm + C::U, C::TILE, row, 2 * quarter + g, x);
        }
        go();
        if (warp == 0) {
            // rows 0 .. 63: dY U^T, rows 64 ..: dZ U^T; where dY is one plane, dZ's second goes into a sum of its own
            issue_ss<PI, PM, PM, true, true, KD / 16, B_ALL, 4>(tb + C::R1, IY, C::TILE, C::DZ - C::DY, IU, C::TILE, vsteps, kTok, false);
            if (C::REST) issue_ss<1, 1, 1, true, true, KD / 16, B_ALL, 4>(tb + C::R0, IY + C::TILE, C::TILE, C::DZ - C::DY, IU, C::TILE, vsteps, kTok, false);
            if (!C::ROOM) issue_ss<PI, PI, PI, true, true, KD / 16, B_ALL, 4>(tb + C::R2, IY, C::TILE, C::K - C::DY, IK, C::TILE, ksteps, kTok, false);    // rows 64 ..: K K^T
            umma_commit(&ws.bar_a);
        }
        // the gradient behind the chunk in the state's place, while those are formed
        if (C::ROOM) WAIT(&ws.full[1], phase);
        walk_late(&ws, is_late(a, LATE_GRADIENTS, bh, now.chunk, LATE_PRODUCT));
        WAIT(&ws.bar_b, 0);                                  // (two phases a unit)
        tmem_fence_after_sync();
        float inner = columns(D, true);
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) inner += __shfl_xor_sync(~0u, inner, m);
        if (lane == 0) total[warp] = inner;
        go();
        if (warp == 0) {
            issue_ts<PM, PM, PM, true, KD / 16, B_ALL, 4>(tb + C::R5, tb + C::S0, KD / 2, IU, C::TILE, vsteps, kTok, false);            // dS1 u
            umma_commit(&ws.bar_b);
        }
        done();
        if (C::ROOM && more && tid == 0 && !walk_given_up(&ws)) copy_early(then);   // (dY and the state's place are free: their products are through, every thread has read)
        __syncwarp();
        if (!C::ROOM) {                                      // queries take dY's place
            load_tile<T>(sm + C::Q, C::TILE, (const T *)a.q, qk, all, a.L, a.Dk, nv, tid, kGradThreads);
            clear_rows(sm + C::Q, C::TILE, PI, a.Dk, KD, tid, kGradThreads);
            __syncthreads();
        }
        {   // F and E in the lower triangles, where their lanes' rows are tokens, and what they say about the decays
            const int i = row & 63;
            const float Hi = ghi[i], Li = glo[i], bi = -beta[i], scale = warp & 2 ? bi : 1.f;
            float own = 0.f;                                 // of this row's pairs in the quarter, up to a column
#pragma unroll 1
            for (int g = 0; g < 2; ++g) {
                const int c = c0 + 8 * g;
                float x[8], y[8], z[8];
                f2 hj[4], lj[4], ga[4], be[4];
                tmem_ld8(x, lane_r + C::R1 + 8 * g);
                tmem_ld8(y, lane_r + C::R2 + 8 * g);
                if (C::REST) tmem_ld8(z, lane_r + C::R0 + 8 * g);
                shared8(hj, ghi + c);
                shared8(lj, glo + c);
                tmem_wait_ld();
                if (!C::ROOM && !(warp & 2)) {               // Q K^T with its ratios: P
                    const unsigned char *P = a.images + at * ((C::PA + PM) * kMatrix) + C::PA * kMatrix;
                    for (int q = 0; q < PM; ++q) HN_G(P + q * kMatrix + image_at(i, c >> 3), 16);
                    image8<PM>(y, P, kMatrix, i, c >> 3);
                }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float r = ratio(Hi, Li, e & 1 ? hj[e / 2].y : hj[e / 2].x, e & 1 ? lj[e / 2].y : lj[e / 2].x);
                    if (C::REST && (warp & 2)) x[e] += z[e];
                    const float plain = x[e];
                    x[e] = c + e < i || (c + e == i && !(warp & 2)) ? r * x[e] : 0.f;
                    z[e] = c + e <= i ? own * scale : 0.f;
                    own = c + e < i ? fmaf(C::ROOM || (warp & 2) ? x[e] : plain, y[e], own) : own;
                    x[e] *= scale;
                }
                planes8_to_image<PM>(sm + (warp & 2 ? C::DZ : C::A), kMatrix, i, c >> 3, x);
                const float before = column_sum8(z, lane);
                if (!(lane & 3)) sums[3][warp & 3][c + (lane >> 2)] = before;
                // dQ and the erased part of dK, as far as they come from the state: F k and E k are added to them
                f2 p[4], q[4];
                tmem_ld8(p, lane_r + C::R4 + 8 * g);
                tmem_ld8(q, lane_r + C::R3 + 8 * g);
                shared8(ga, gamma + c);
                shared8(be, gates + 3 * kTok + c);
                if (row < KD) {
                    image8<PI>(x, sm + C::Q, C::TILE, row, c >> 3);
                    image8<PI>(y, sm + C::K, C::TILE, row, c >> 3);
                }
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = mul2(p[e], ga[e]);
                    q[e] = mul2(q[e], be[e]);
                    const f2 both = fma2(q[e], make2(y[2 * e], y[2 * e + 1]), mul2(p[e], make2(x[2 * e], x[2 * e + 1])));
                    z[2 * e] = row < a.Dk ? both.x : 0.f;    // (a lane without a channel holds whatever lay behind an image)
                    z[2 * e + 1] = row < a.Dk ? both.y : 0.f;
                }
                tmem_st8(lane_r + C::R4 + 8 * g, p);
                tmem_st8(lane_r + C::R3 + 8 * g, q);
                const float state = column_sum8(z, lane);
                if (!(lane & 3)) sums[1][warp & 3][c + (lane >> 2)] = state;
            }
            pairs[quarter][row] = own;
        }
        uint4 ks[2];
        if (C::ROOM && row < KD)
#pragma unroll
            for (int g = 0; g < 2; ++g) ks[g] = *(const uint4 *)(sm + C::K + image_at(row, 2 * quarter + g));
        go();
        if (warp == 0) {
            issue_ss<PI, PM, PM, false, false, kTok / 16, B_LOWER>(tb + C::R4, IK, C::TILE, 0, IA, kMatrix, kTok / 16, kTok, true);             // F k
            issue_ss<PI, PM, PM, false, false, kTok / 16, B_LOWER>(tb + C::R3, IK, C::TILE, 0, IZ, kMatrix, kTok / 16, kTok, true);             // E k
            issue_ss<PI, PM, PM, false, true, kTok / 16, B_LOWER_T>(tb + C::R2, IQ, C::TILE, 0, IA, kMatrix, kTok / 16, kTok, false);           // F q
            issue_ss<PI, PM, PM, false, true, kTok / 16, B_LOWER_T>(tb + C::R2, IK, C::TILE, 0, IZ, kMatrix, kTok / 16, kTok, true);            // E k, the other way
            umma_commit(&ws.bar_a);
        }
        WAIT(&ws.bar_b, 1);                                  // (dS1 u: in front of the next unit's wait for it)
        done();
        if (C::ROOM && more && tid == 0 && !walk_given_up(&ws)) copy_rest(then, phase ^ 1);     // (every product is through, and what the threads read they have)
        __syncwarp();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int c = c0 + 8 * g;
            const bool in = row < a.Dk;
            float x[8], y[8], z[8], w[8], u[8];
            f2 de[4];
            tmem_ld8(x, lane_r + C::R4 + 8 * g);             // dQ of this head
            tmem_ld8(y, lane_r + C::R3 + 8 * g);
            tmem_ld8(w, lane_r + C::R2 + 8 * g);
            tmem_ld8(u, lane_r + C::R5 + 8 * g);
            shared8(de, delta + c);
            if (C::ROOM) bf16_widen8(z, ks[g]);
            else if (row < KD) image8<PI>(z, sm + C::K, C::TILE, row, c >> 3);
            tmem_wait_ld();
            if (walk_given_up(&ws))
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = y[e] = kLost;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] *= e & 1 ? de[e / 2].y : de[e / 2].x;
                dq[g][e] += x[e];
                dk[g][e] += y[e] + (w[e] + u[e]);
                x[e] = in ? u[e] * z[e] : 0.f;
            }
            const float sum = column_sum8(x, lane);
            if (!(lane & 3)) sums[2][warp & 3][c + (lane >> 2)] = sum;
            if (last) {                                      // U is through: dK into half of its place
                if (C::ROOM && a.copies) {
                    if (row < KD) {
                        *(uint4 *)(sm + C::OUT + image_at(row, 2 * quarter + g)) = bf16_8(dq[g], now.n - t - 8 * g);
                        *(uint4 *)(sm + C::U + C::TILE + image_at(row, 2 * quarter + g)) = bf16_8(dk[g], now.n - t - 8 * g);
                    }
                } else if (in && t + 8 * g < a.L) {
                    const long long to = (now.bk * a.Dk + row) * a.L + t + 8 * g;
                    store8<T>((T *)a.dq, to, a.L, a.L - t - 8 * g, now.n - t - 8 * g, dq[g]);
                    store8<T>((T *)a.dk, to, a.L, a.L - t - 8 * g, now.n - t - 8 * g, dk[g]);
                }
            }
        }
        fence_async_smem();
        tmem_fence_before_sync();
        __syncthreads();                                     // images, sums and tensor memory have been read, results written
        tmem_fence_after_sync();
        if (tid == 128) {
            if (last && C::ROOM && a.copies) {
                tma_store_3d(&maps.out, sm + C::OUT, t0, 0, (int)now.bk);
                tma_store_3d(&maps.outk, sm + C::U + C::TILE, t0, 0, (int)now.bk);
                tma_commit();
                tma_wait_read0();                            // (U is formed anew behind the next barriers)
            }
            if (!C::ROOM && more && !walk_given_up(&ws)) {
                copy_early(then);
                copy_rest(then, phase ^ 1);
            }
        }
        __syncwarp();
        if (warp < 2) {                                      // two tokens a lane; warp 0: the decays, warp 1: beta
            float s[2];
            auto token = [&](int what, int i) { return (sums[what][0][i] + sums[what][1][i]) + (sums[what][2][i] + sums[what][3][i]); };
            if (warp == 0) {
                // what crosses a token: pairs of a query or an erasure from it on and a value before it (in the quarter of the earlier token's
                // column: summed above; in the quarters before), the state before the chunk and tokens from it on, the gradient behind the
                // chunk and tokens before it, the state before the chunk and the gradient behind it.  Every sum runs towards its larger terms
                float c[2], d[2], in[3][2], rest[4], front;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i = 2 * lane + e;
                    c[e] = token(1, i);
                    d[e] = token(2, i);
                    s[e] = token(3, i);
                    float up = 0.f;                          // row i's pairs in the quarters 0 .. q
#pragma unroll
                    for (int q = 0; q < 3; ++q) in[q][e] = up += fmaf(-beta[i], pairs[q][kTok + i], pairs[q][i]);
                }
                rest[0] = c[0] + c[1];
#pragma unroll
                for (int q = 0; q < 3; ++q) rest[q + 1] = in[q][0] + in[q][1];
                front = d[0] + d[1];
#pragma unroll
                for (int m = 1; m < 32; m <<= 1) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float o = __shfl_down_sync(~0u, rest[q], m);
                        if (lane + m < 32) rest[q] += o;
                    }
                    const float o = __shfl_up_sync(~0u, front, m);
                    if (lane >= m) front += o;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) { const float o = __shfl_down_sync(~0u, rest[q], 1); rest[q] = lane < 31 ? o : 0.f; }
                const float o = __shfl_up_sync(~0u, front, 1);
                front = lane ? o : 0.f;
                float w = lane < 16 ? gamma[kTok - 1] * total[lane] : 0.f;
#pragma unroll
                for (int m = 1; m < 16; m <<= 1) w += __shfl_xor_sync(~0u, w, m);
                w = __shfl_sync(~0u, w, 0);
                const int quarter_of = lane >> 3;
#pragma unroll
                for (int e = 1; e >= 0; --e) {
                    rest[0] += c[e];
                    float before = 0.f;
#pragma unroll
                    for (int q = 0; q < 3; ++q) {
                        rest[q + 1] += in[q][e];
                        if (quarter_of == q + 1) before = rest[q + 1];
                    }
                    s[e] += before + rest[0] + (e ? front + d[0] : front) + w;
                }
            } else
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int i = 2 * lane + e;
                    s[e] = token(0, i) - ((pairs[0][kTok + i] + pairs[1][kTok + i]) + (pairs[2][kTok + i] + pairs[3][kTok + i]));
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = 2 * lane + e;
                if (walk_given_up(&ws)) s[e] = kLost;
                if (i >= room) continue;
                if (warp == 1) { HN_G(a.dbeta + grow + i, 4); a.dbeta[grow + i] = i < nv ? s[e] : 0.f; }
                else if (a.dg) {
                    float d = s[e];
                    if (a.decay == DELTA_SIGMOID && i < nv) { HN_G(a.g + grow + i, 4); d /= 1.f + expf(__ldg(a.g + grow + i)); }
                    HN_G(a.dg + grow + i, 4);
                    a.dg[grow + i] = i < nv ? d : 0.f;
                }
            }
        }
    }
    tmem_fence_before_sync();
    walk_end(&ws, 3, &hn_delta_backward_status, warp, 0);
    if (warp == 0) tmem_dealloc(tb, 512);
    pdl_trigger();                                           // (late: see delta.cuh)
}

// ---- host -----------------------------------------------------------------------------------------------------------

int delta_backward_status()
{
    int v = 0;
    return cudaMemcpyFromSymbol(&v, hn_delta_backward_status, sizeof(int)) == cudaSuccess ? v : -1;
}

template <typename T, int KD> static int launch_back(DeltaArgs a, cudaStream_t st)
{
    DeltaMaps m{};
    a.copies = delta_maps<T>(m, a, KD, a.dy, a.dv, nullptr);
    const long long blocks = (long long)a.B * a.H * a.segments;
    if (a.segments > 1) {
        if (const int e = launch_delta<delta_walk_back_kernel<T, KD, WALK_MAPS>>(a, 2 * blocks, kWalkThreads, WalkBack<T, KD>::BYTES, st, m)) return e;
        if (const int e = launch_delta_join(a, a.ds_end, true, st)) return e;
    }
    if (const int e = launch_delta<delta_walk_back_kernel<T, KD, WALK_RUN>>(a, blocks, kWalkThreads, WalkBack<T, KD>::BYTES, st, m)) return e;
    a.copies = delta_maps<T>(m, a, KD, a.dy, a.dq, a.dk);
    const long long items = (long long)a.B * a.Hk * a.chunks;
    return launch_delta<delta_gradients_kernel<T, KD>>(a, items < kSms ? items : kSms, kGradThreads, Grads<T, KD>::BYTES, st, m);
}
int launch_delta_backward(const DeltaArgs &a, int dtype, cudaStream_t st)
{
    if (const int e = launch_delta_prepare(a, dtype, st)) return e;
    const bool small = a.Dk <= 64 && a.Dv <= 64;
    if (dtype == HYENAND_F32) return small ? launch_back<float, 64>(a, st) : launch_back<float, 128>(a, st);
    return small ? launch_back<bf16, 64>(a, st) : launch_back<bf16, 128>(a, st);
}

}  // namespace hn
