// The gated delta rule in chunks of 64 tokens: what its kernels share (internal).
//
// For one value head, S in R^{Dv x Dk}:   u_t = beta_t (v_t - a_t S_{t-1} k_t),   S_t = a_t S_{t-1} + u_t k_t^T,   y_t = S_t q_t.
// Over a chunk that starts from S0, with G_i = log a_1 + .. + log a_i, gamma_i = exp(G_i), delta_i = exp(G_64 - G_i), r_ij = exp(G_i - G_j):
//     T_ij = beta_i r_ij (k_i . k_j)  (j < i),   A = (I + T)^{-1},   P_ij = r_ij (q_i . k_j)  (j <= i),
//     R_i = v_i - gamma_i S0 k_i,   U = A (beta R),   Y_i = gamma_i S0 q_i + sum_j P_ij u_j,   S1 = gamma_64 S0 + sum_j delta_j u_j k_j^T.
// Gradient, from dY and dS1:
//     dU_j = sum_i P_ij dY_i + delta_j dS1 k_j,   dZ = A^T dU,   dV = beta dZ,
//     dS0 = gamma_64 dS1 + sum_i gamma_i (dY_i q_i^T - beta_i dZ_i k_i^T),
//     F_ij = r_ij (dY_i . u_j)  (j <= i),   E_ij = - beta_i r_ij (dZ_i . u_j)  (j < i),
//     dQ_i = gamma_i S0^T dY_i + sum_j F_ij k_j,
//     dK_i = [sum_j E_ij k_j - gamma_i beta_i S0^T dZ_i]  +  [sum_j (F_ji q_j + E_ji k_j) + delta_i dS1^T u_i]      (erased, written),
//     dbeta_i = dZ_i . R_i - sum_{j<i} (dZ_i . u_j) r_ij (k_i . k_j),
//     d log a_t = sum_{i >= t > j} [F_ij (q_i . k_j) + E_ij (k_i . k_j)]  +  sum_{i >= t} gamma_i [q_i . S0^T dY_i - beta_i k_i . S0^T dZ_i]
//                 +  sum_{j < t} delta_j k_j . dS1^T u_j  +  gamma_64 <S0, dS1>.
// (What crosses token t carries a_t and nothing else does.  The same as a running sum of q dQ + k dK, erased less written, is a difference of
// numbers of order 1: right to 1e-3 of itself at log a = -8, to nothing at -16.)
//
// The products run on the tensor cores in bf16 with fp32 sums.  A number that is no bf16 value goes in as a sum of bf16 values ("planes"):
// two for bf16 tensors (16 bits, errors of 2^-17: states and sums are fp32 and a result is rounded once, so these errors stay far
// below a bf16 result's own), three for fp32 tensors (24 bits).  Tensors of bf16 are one plane as they are.  A product of planes
// p and q is formed where p + q is below the number of planes.  A has three planes always: with keys that repeat its entries are as large
// as beta and the same along its diagonals, their roundings too, and what is summed of A Z over a chunk cancels (512 tokens with one key at
// beta = 2: with two planes a state was off by 1.8e-2, with three by 1.8e-4, 7e-5 from fp32 tensors.  Two products more on the chain:
// a walk of 64 chunks 236 -> 241 us, back 255 -> 263).
#pragma once
#include "entry.cuh"
#include "octet.cuh"
#include "pair.cuh"
#include "umma.cuh"

namespace hn {

constexpr int kTok = 64;                                  // tokens of a chunk
enum { DELTA_LOG = HYENAND_DECAY_LOG, DELTA_SIGMOID = HYENAND_DECAY_SIGMOID, DELTA_NONE = HYENAND_DECAY_NONE };

template <typename T> struct Planes { static constexpr int IN = 1, MID = 2, INVERSE = 3; };
template <> struct Planes<float> { static constexpr int IN = 3, MID = 3, INVERSE = 3; };
constexpr int kMatrix = kTok * 128;                       // bytes of one plane of a 64 x 64 matrix
// floats of a chunk: gamma, delta, beta, -beta gamma, what carries the state (see Carry), and G in two parts (see ratio)
constexpr int kGates = 6 * kTok + 4, kCarry = 4 * kTok, kSums = kCarry + 4;
constexpr int kWalkGates = kCarry * 4;                    // bytes of the first four

struct DeltaArgs {
    const void *q, *k, *v;
    const float *g, *beta, *s0;
    const int *lengths;
    void *y;
    float *s_end, *marks;
    // gradient
    const void *dy;
    const float *ds_end;
    void *dq, *dk, *dv;
    float *dg, *dbeta, *ds0;
    // workspace
    unsigned char *images;                                // [B H][chunks]: planes of A, planes of P
    float *gates;                                         // [B H][chunks][kGates]
    float *maps, *starts;                                 // [B H][segments][Dv + Dk][map_pitch], [B H][segments] states as kept
    float *dstates, *dz;                                  // [B H][chunks] states as kept, [B H][chunks][Dv][64]
    int B, H, Hk, L, Dk, Dv, decay, chunks, segments, per_segment;
    int copies;                                           // 1: tiles come as tensor copies
#ifdef HYENAND_DEBUG
    int late_kernel, late_chunk, late_wait;               // the wait of head 0 that is taken to run out (late_kernel < 0: none)
#endif
};
// The kernels whose waits the checked build can take to run out, and which wait of a chunk (of a segment, in the join): for copies; for a
// product, by the threads that go on from it; for a product, by those that store it
enum { LATE_PREPARE, LATE_WALK, LATE_MAPS, LATE_JOIN, LATE_BACK, LATE_BACK_MAPS, LATE_GRADIENTS };
enum { LATE_COPIES, LATE_PRODUCT, LATE_RESULT };
#ifdef HYENAND_DEBUG
__device__ __forceinline__ bool is_late(const DeltaArgs &a, int kernel, long long head, int chunk, int wait)
{
    return a.late_kernel == kernel && head == 0 && a.late_chunk == chunk && a.late_wait == wait;
}
#else
__device__ __forceinline__ bool is_late(const DeltaArgs &, int, long long, int, int) { return false; }
#endif

__host__ __device__ __forceinline__ int map_pitch(int Dk) { return (Dk + 3) & ~3; }

__device__ __forceinline__ int live_tokens(const DeltaArgs &a, int b)
{
    if (!a.lengths) return a.L;
    HN_G(a.lengths + b, 4);
    const int n = __ldg(a.lengths + b);
    return n < 0 ? 0 : n < a.L ? n : a.L;
}

// eight columns of this thread's lane
__device__ __forceinline__ void tmem_ld8(float (&v)[8], unsigned at)
{
    unsigned u[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]) : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void tmem_st8(unsigned at, const float (&v)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n"
                 ::"r"(at), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])),
                   "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])) : "memory");
}
// (not "memory": loads of shared memory behind it may go ahead; the wait for stores is)
__device__ __forceinline__ void tmem_st4(unsigned at, const unsigned (&v)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]));
}

// a pair of numbers as PM planes of bf16 pairs, each the rest of the ones before, rounded to nearest (so that a rest has either sign
// and what is left out of a product, rest times rest, averages out: cut off instead, states were off by 7e-6, now by 2e-6)
template <int PM> __device__ __forceinline__ void split_pair(f2 x, unsigned (&w)[PM])
{
#pragma unroll
    for (int p = 0; p < PM; ++p) {
        const __nv_bfloat162 r = __float22bfloat162_rn(x);
        w[p] = *(const unsigned *)&r;
        if (p + 1 < PM) x = fma2(make2(__uint_as_float(w[p] << 16), __uint_as_float(w[p] & 0xffff0000u)), pair(-1.f), x);
    }
}
template <int PM> __device__ __forceinline__ void split_pair(float x, float y, unsigned (&w)[PM]) { split_pair<PM>(make2(x, y), w); }

// 2 C numbers of this thread's row as the A operand in tensor memory: C columns per plane, planes `pitch` columns apart
template <int PM, int C> __device__ __forceinline__ void planes_to_tmem(unsigned at, int pitch, const f2 (&x)[C])
{
    float w[PM][C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        unsigned u[PM];
        split_pair<PM>(x[i], u);
#pragma unroll
        for (int p = 0; p < PM; ++p) w[p][i] = __uint_as_float(u[p]);
    }
#pragma unroll
    for (int p = 0; p < PM; ++p) TmemIO<C>::st(at + p * pitch, w[p]);
}
// 32 columns of this thread's lane, in pairs
__device__ __forceinline__ void tmem_ld(f2 (&v)[16], unsigned at)
{
    float x[32];
    TmemIO<32>::ld(x, at);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = make2(x[2 * i], x[2 * i + 1]);
}
// the same eight columns at a time
__device__ __forceinline__ void tmem_ld8(f2 (&v)[4], unsigned at)
{
    float x[8];
    tmem_ld8(x, at);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make2(x[2 * i], x[2 * i + 1]);
}
__device__ __forceinline__ void tmem_st8(unsigned at, const f2 (&v)[4])
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split2(v[i], x[2 * i], x[2 * i + 1]);
    tmem_st8(at, x);
}
template <int PM> __device__ __forceinline__ void planes8_to_tmem(unsigned at, int pitch, const f2 (&x)[4])
{
    unsigned w[PM][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned u[PM];
        split_pair<PM>(x[i], u);
#pragma unroll
        for (int p = 0; p < PM; ++p) w[p][i] = u[p];
    }
#pragma unroll
    for (int p = 0; p < PM; ++p) tmem_st4(at + p * pitch, w[p]);
}
// 16 columns of this thread's lane, on their way until the next wait for loads
struct Sixteen {
    float x[16];
    __device__ __forceinline__ void load(unsigned at) { TmemIO<16>::ld(x, at); }
    __device__ __forceinline__ f2 get(int i) const { return make2(x[2 * i], x[2 * i + 1]); }
};
// What a chunk leaves of a state, gamma_64 S = keep S + by S: a decay next to 1 as S + (gamma_64 - 1) S, where only the sum rounds the
// state, with either sign.  As a factor, it is off by up to half a step in every chunk alike: at g = -1e-6 a state of 262144 tokens was off by
// 7e-5.  Below a half there is nothing to lose: 0 S + gamma_64 S.
struct Carry {
    f2 keep, by;
    __device__ __forceinline__ explicit Carry(const float *two) { const float2 c = *(const float2 *)two; keep = pair(c.x); by = pair(c.y); }
};
// S = gamma_64 S + gain (this thread's columns of both, eight pairs at a time, the next loads under way), and S as an operand again
template <int PM, int C> __device__ __forceinline__ void state_onwards(f2 (&S)[C], const Carry &carry, unsigned gain, unsigned planes, int pitch)
{
    Sixteen g[2];
    g[0].load(gain);
#pragma unroll
    for (int b = 0; b < C / 8; ++b) {
        tmem_wait_ld();
        if (b + 1 < C / 8) g[(b + 1) & 1].load(gain + 16 * (b + 1));
        f2 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = S[8 * b + j] = fma2(carry.keep, S[8 * b + j], fma2(carry.by, S[8 * b + j], g[b & 1].get(j)));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f2 y[4] = {x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
            planes8_to_tmem<PM>(planes + 8 * b + 4 * j, pitch, y);
        }
    }
}
// eight numbers of shared memory
__device__ __forceinline__ void shared8(f2 (&v)[4], const float *p)
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    v[0] = make2(a.x, a.y); v[1] = make2(a.z, a.w); v[2] = make2(b.x, b.y); v[3] = make2(b.z, b.w);
}
// eight numbers as planes: into tensor memory (four columns each), into chunk `chunk` of row `row` of an image
template <int PM> __device__ __forceinline__ void planes8_to_tmem(unsigned at, int pitch, const float (&x)[8])
{
    unsigned w[PM][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned u[PM];
        split_pair<PM>(x[2 * i], x[2 * i + 1], u);
#pragma unroll
        for (int p = 0; p < PM; ++p) w[p][i] = u[p];
    }
#pragma unroll
    for (int p = 0; p < PM; ++p) tmem_st4(at + p * pitch, w[p]);
}
template <int PM> __device__ __forceinline__ void planes8(uint4 (&w)[PM], const float (&x)[8])
{
    unsigned u[4][PM];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_pair<PM>(x[2 * i], x[2 * i + 1], u[i]);
#pragma unroll
    for (int p = 0; p < PM; ++p) w[p] = make_uint4(u[0][p], u[1][p], u[2][p], u[3][p]);
}
template <int PM> __device__ __forceinline__ void planes8_to_image(unsigned char *image, int pitch, int row, int chunk, const float (&x)[8])
{
    uint4 w[PM];
    planes8<PM>(w, x);
#pragma unroll
    for (int p = 0; p < PM; ++p) *(uint4 *)(image + p * pitch + image_at(row, chunk)) = w[p];
}
template <int PI> __device__ __forceinline__ void image8(float (&x)[8], const unsigned char *image, int pitch, int row, int chunk)
{
#pragma unroll
    for (int p = PI - 1; p >= 0; --p) {
        const uint4 w = *(const uint4 *)(image + p * pitch + image_at(row, chunk));
        const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = __uint_as_float(u[i] << 16), hi = __uint_as_float(u[i] & 0xffff0000u);
            x[2 * i] = p == PI - 1 ? lo : x[2 * i] + lo;
            x[2 * i + 1] = p == PI - 1 ? hi : x[2 * i + 1] + hi;
        }
    }
}
__device__ __forceinline__ void bf16_widen8(float (&x)[8], uint4 w)
{
    const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}

// ---- tensors in device memory ---------------------------------------------------------------------------------------

// 16 bytes from element `at` of a tensor of n elements whose rows do not start on 16 bytes: cut out of two words
__device__ __forceinline__ uint4 load_unaligned(const bf16 *p, long long at, long long n)
{
    const int s = (int)(at & 7);
    const bf16 *base = p + (at - s);
    if (at - s + (s ? 16 : 8) > n) {                      // (the tensor's last words: element by element)
        unsigned u[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < n) { HN_G(p + at + i, 2); u[i >> 1] |= (unsigned)__ldg((const unsigned short *)p + at + i) << (16 * (i & 1)); }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    HN_G(base, 16);
    const uint4 a = __ldg((const uint4 *)base);
    if (!s) return a;
    HN_G(base + 8, 16);
    const uint4 b = __ldg((const uint4 *)base + 1);
    unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, o[5];
    const int ws = s >> 1;
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = ws == 0 ? w[i] : ws == 1 ? w[i + 1] : ws == 2 ? w[i + 2] : w[i + 3];
    const int sh = (s & 1) * 16;
    return make_uint4(__funnelshift_r(o[0], o[1], sh), __funnelshift_r(o[1], o[2], sh), __funnelshift_r(o[2], o[3], sh), __funnelshift_r(o[3], o[4], sh));
}
// all but the first n (0 .. 8) of eight bf16 values replaced by zero
__device__ __forceinline__ uint4 keep_first(uint4 w, int n)
{
    const unsigned half = (n & 1) ? 0xffffu : 0u;
    const int full = n >> 1;
    w.x = full > 0 ? w.x : full == 0 ? w.x & half : 0u;
    w.y = full > 1 ? w.y : full == 1 ? w.y & half : 0u;
    w.z = full > 2 ? w.z : full == 2 ? w.z & half : 0u;
    w.w = full > 3 ? w.w : full == 3 ? w.w & half : 0u;
    return w;
}

// A chunk's tile of a tensor as images: `rows` rows of [.][L] from element `at` (row 0, the chunk's first token), the first nv of 64
// tokens of each, zero behind them; `threads` threads together.  Rows behind `rows` are the caller's.
template <typename T> __device__ __forceinline__ void load_tile(unsigned char *image, int pitch, const T *p, long long at, long long n, int L, int rows, int nv, int tid, int threads)
{
    constexpr int V = sizeof(T) == 2 ? 4 : 2;             // vectors of eight tokens in flight
    const bool aligned = sizeof(T) == 2 ? L % 8 == 0 : L % 4 == 0;
    for (int i0 = tid; i0 < rows * 8; i0 += threads * V) {
        if constexpr (sizeof(T) == 2) {
            uint4 w[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int i = i0 + j * threads, row = i >> 3, c = i & 7, left = nv - c * 8;
                w[j] = make_uint4(0, 0, 0, 0);
                if (i >= rows * 8 || left <= 0) continue;
                const long long e = at + (long long)row * L + c * 8;
                if (aligned) { HN_G((const bf16 *)p + e, 16); w[j] = __ldg((const uint4 *)((const bf16 *)p + e)); }
                else w[j] = load_unaligned((const bf16 *)p, e, n);
                if (left < 8) w[j] = keep_first(w[j], left);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int i = i0 + j * threads;
                if (i < rows * 8) *(uint4 *)(image + image_at(i >> 3, i & 7)) = w[j];
            }
        } else {
            float x[V][8];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int i = i0 + j * threads, row = i >> 3, c = i & 7, left = nv - c * 8;
#pragma unroll
                for (int t = 0; t < 8; ++t) x[j][t] = 0.f;
                if (i >= rows * 8 || left <= 0) continue;
                const long long e = at + (long long)row * L + c * 8;
                if (aligned && left >= 8) {
                    HN_G((const float *)p + e, 32);
                    const float4 lo = __ldg((const float4 *)((const float *)p + e)), hi = __ldg((const float4 *)((const float *)p + e) + 1);
                    x[j][0] = lo.x; x[j][1] = lo.y; x[j][2] = lo.z; x[j][3] = lo.w; x[j][4] = hi.x; x[j][5] = hi.y; x[j][6] = hi.z; x[j][7] = hi.w;
                } else {
#pragma unroll
                    for (int t = 0; t < 8; ++t)
                        if (t < left) x[j][t] = IO<float>::ld((const float *)p, e + t);
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int i = i0 + j * threads;
                if (i >= rows * 8) continue;
                unsigned u[4][3];
#pragma unroll
                for (int t = 0; t < 4; ++t) split_pair<3>(x[j][2 * t], x[j][2 * t + 1], u[t]);
#pragma unroll
                for (int q = 0; q < 3; ++q) *(uint4 *)(image + q * pitch + image_at(i >> 3, i & 7)) = make_uint4(u[0][q], u[1][q], u[2][q], u[3][q]);
            }
        }
    }
}
// rows `from` .. `to` of an image's planes: zero
__device__ __forceinline__ void clear_rows(unsigned char *image, int pitch, int planes, int from, int to, int tid, int threads)
{
    for (int p = 0; p < planes; ++p)
        for (int i = from * 8 + tid; i < to * 8; i += threads) *(uint4 *)(image + p * pitch + i * 16) = make_uint4(0, 0, 0, 0);
}

// 32 tokens of one row of fp32 values; zero behind the first nv
__device__ __forceinline__ void load_row(f2 (&x)[16], const float *p, long long at, int L, int nv)
{
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (L % 4 == 0 && nv >= 4 * c + 4) {
            HN_G(p + at + 4 * c, 16);
            const float4 w = __ldg((const float4 *)(p + at) + c);
            x[2 * c] = make2(w.x, w.y);
            x[2 * c + 1] = make2(w.z, w.w);
        } else {
#pragma unroll
            for (int i = 2 * c; i < 2 * c + 2; ++i)
                x[i] = make2(2 * i < nv ? IO<float>::ld(p, at + 2 * i) : 0.f, 2 * i + 1 < nv ? IO<float>::ld(p, at + 2 * i + 1) : 0.f);
        }
    }
}
// eight tokens of one row, the first `room` of them; from the nv-th on they are zero
template <typename T> __device__ __forceinline__ void store8(T *p, long long at, int L, int room, int nv, const float (&x)[8])
{
    constexpr int V = 16 / sizeof(T);
    if (L % V == 0) {
#pragma unroll
        for (int c = 0; c < 8 / V; ++c) {
            if (c * V >= room) break;
            uint4 w;
            T *e = (T *)&w;
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = (T)(c * V + i < nv ? x[c * V + i] : 0.f);
            HN_G(p + at + c * V, 16);
            *(uint4 *)(p + at + c * V) = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < room) IO<T>::st(p, at + i, i < nv ? x[i] : 0.f);
    }
}
__device__ __forceinline__ uint4 bf16_8(const float (&x)[8], int nv)
{
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(2 * i < nv ? x[2 * i] : 0.f, 2 * i + 1 < nv ? x[2 * i + 1] : 0.f);
        u[i] = *(const unsigned *)&r;
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// A state that stays inside the library (marks, the gradient behind a chunk): column quartets [D / 4][rows], the rows of a group of eight
// exchanged by the quartet.  Threads that hold rows write and read it in whole lines; from shared memory both rows and columns come
// without bank conflicts.
__host__ __device__ __forceinline__ int kept_rows(int rows) { return (rows + 7) & ~7; }
__host__ __device__ __forceinline__ long long kept_floats(int rows, int D) { return (long long)kept_rows(rows) * ((D + 3) & ~3); }
__device__ __forceinline__ int kept_at(int row, int quartet, int rows8) { return quartet * rows8 + (row ^ (quartet & 7)); }
// (columns 4 FROM .. 4 TO - 1 of this thread's 2 C from `col`, a multiple of 32)
template <int FROM, int TO, int C> __device__ __forceinline__ void keep_state(float *p, const f2 (&s)[C], int row, int rows, int col, int D)
{
    const int rows8 = kept_rows(rows);
    if (row >= rows8) return;
    float4 *to = (float4 *)p + ((col >> 2) + FROM) * rows8;
#pragma unroll
    for (int i = FROM; i < TO; ++i) {
        if (col + 4 * i >= D) break;
        HN_G(to + (row ^ (i & 7)), 16);
        to[row ^ (i & 7)] = make_float4(s[2 * i].x, s[2 * i].y, s[2 * i + 1].x, s[2 * i + 1].y);
        to += rows8;
    }
}
template <int C> __device__ __forceinline__ void load_kept(float (&s)[C], const float *p, int row, int rows, int col, int D)
{
    const int rows8 = kept_rows(rows);
#pragma unroll
    for (int i = 0; i < C; i += 4) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < rows8 && col + i < D) {
            const float4 *from = (const float4 *)p + kept_at(row, (col + i) >> 2, rows8);
            HN_G(from, 16);
            w = *from;
        }
        s[i] = w.x; s[i + 1] = w.y; s[i + 2] = w.z; s[i + 3] = w.w;
    }
}
// this thread's C columns from `col` of row `row` of a state [rows][D], zero outside it
template <int C> __device__ __forceinline__ void load_state(float (&s)[C], const float *p, int row, int rows, int col, int D)
{
    if (row < rows && D % 4 == 0) {
#pragma unroll
        for (int i = 0; i < C; i += 4) {
            float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
            if (col + i < D) { HN_G(p + (long long)row * D + col + i, 16); w = *(const float4 *)(p + (long long)row * D + col + i); }
            s[i] = w.x; s[i + 1] = w.y; s[i + 2] = w.z; s[i + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            s[i] = 0.f;
            if (row < rows && col + i < D) { HN_G(p + (long long)row * D + col + i, 4); s[i] = p[(long long)row * D + col + i]; }
        }
    }
}
template <int C> __device__ __forceinline__ void store_state(float *p, const float (&s)[C], int row, int rows, int col, int D)
{
    if (row >= rows) return;
    if (D % 4 == 0) {
#pragma unroll
        for (int i = 0; i < C; i += 4)
            if (col + i < D) { HN_G(p + (long long)row * D + col + i, 16); *(float4 *)(p + (long long)row * D + col + i) = make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]); }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (col + i < D) { HN_G(p + (long long)row * D + col + i, 4); p[(long long)row * D + col + i] = s[i]; }
    }
}


// ---- a chunk's decays ---------------------------------------------------------------------------------------------------

// log a.  Below -110 the factor is zero in fp32: the sum of a chunk stays small enough for differences.  A NaN stays one.
__device__ __forceinline__ float log_decay(float g, int decay)
{
    if (decay == DELTA_NONE) return 0.f;
    float x = g;
    if (decay == DELTA_SIGMOID) x = g >= 0.f ? -log1pf(expf(-g)) : g - log1pf(expf(g));
    return x < -110.f ? -110.f : x;
}
// G of a chunk's 64 tokens, by one warp, summed in 64 bits (differences of neighbours beside a sum of many) and kept in units of log 2 as a
// float and the rest; tokens from nv on decay nothing
__device__ __forceinline__ void chunk_sums(float *hi, float *lo, const float *g, int decay, int nv, int lane)
{
    double x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = 2 * lane + i;
        x[i] = 0.;
        if (decay != DELTA_NONE && t < nv) { HN_G(g + t, 4); x[i] = log_decay(__ldg(g + t), decay); }
    }
    double s = x[0] + x[1];
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        const double o = __shfl_up_sync(~0u, s, m);
        if (lane >= m) s += o;
    }
    const double G[2] = {(s - x[1]) * 1.4426950408889634, s * 1.4426950408889634};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        hi[2 * lane + i] = (float)G[i];
        lo[2 * lane + i] = (float)(G[i] - (float)G[i]);
    }
}
// exp(G_i - G_j)
__device__ __forceinline__ float ratio(float hi, float lo, float hj, float lj) { return ex2((hi - hj) + (lo - lj)); }

// ---- products ------------------------------------------------------------------------------------------------------------

// The rows of B that a product needs at step k of its contraction: all of them; for a lower triangle of 64 x 64 taken by rows (i >= j)
// those from 16 k on, taken by columns (j <= i) those below 16 (k + 1)
enum { B_ALL = 0, B_LOWER = 1, B_LOWER_T = 2 };

// d (+)= sum of the products of planes p of A (tensor memory, `pa` columns apart) and q of B (images, `pb` bytes apart), p < NA, q < NB,
// p + q < MAX, over the first `steps` of STEPS 16-steps; the smallest first (the sums are cut off, not rounded, at every instruction)
template <int NA, int NB, int MAX, bool BCOLS, int STEPS, int PART = B_ALL, int UNROLL = STEPS>
__device__ __forceinline__ void issue_ts(unsigned d, unsigned a, int pa, unsigned b, int pb, int steps, int n, bool add, unsigned next = 1024)
{
#pragma unroll
    for (int sum = MAX - 1; sum >= 0; --sum)
#pragma unroll
        for (int p = 0; p <= sum; ++p)
            if (const int q = sum - p; p < NA && q < NB) {
                const unsigned A = a + p * pa, B = BCOLS ? umma_cols(b + q * pb, next) : umma_rows(b + q * pb);
#pragma unroll UNROLL
                for (int e = 0; e < STEPS; ++e) {
                    const int k = PART == B_LOWER_T ? STEPS - 1 - e : e, from = PART == B_LOWER ? 16 * k : 0, cols = PART == B_ALL ? n : PART == B_LOWER ? kTok - 16 * k : 16 * (k + 1);
                    if (PART == B_ALL && k >= steps) break;
                    umma_ts(d + from, A + k * 8, B + k * (BCOLS ? kColStep : kRowStep) + from * (128 >> 4), umma_kind(cols, false, BCOLS), add);
                    add = true;
                }
            }
}
// the same with A in images; `next`: see umma_cols
template <int NA, int NB, int MAX, bool ACOLS, bool BCOLS, int STEPS, int PART = B_ALL, int UNROLL = STEPS>
__device__ __forceinline__ void issue_ss(unsigned d, unsigned a, int pa, unsigned next, unsigned b, int pb, int steps, int n, bool add)
{
#pragma unroll
    for (int sum = MAX - 1; sum >= 0; --sum)
#pragma unroll
        for (int p = 0; p <= sum; ++p)
            if (const int q = sum - p; p < NA && q < NB) {
                const unsigned A = ACOLS ? umma_cols(a + p * pa, next) : umma_rows(a + p * pa), B = BCOLS ? umma_cols(b + q * pb) : umma_rows(b + q * pb);
#pragma unroll UNROLL
                for (int e = 0; e < STEPS; ++e) {
                    const int k = PART == B_LOWER_T ? STEPS - 1 - e : e, from = PART == B_LOWER ? 16 * k : 0, cols = PART == B_ALL ? n : PART == B_LOWER ? kTok - 16 * k : 16 * (k + 1);
                    if (PART == B_ALL && k >= steps) break;
                    umma_ss(d + from, A + k * (ACOLS ? kColStep : kRowStep), B + k * (BCOLS ? kColStep : kRowStep) + from * (128 >> 4), umma_kind(cols, ACOLS, BCOLS), add);
                    add = true;
                }
            }
}

// the warp's number, as a value that the compiler knows to be the same in all its lanes (see umma.cuh)
__device__ __forceinline__ int uniform_warp(int warp) { return __shfl_sync(~0u, warp, 0); }

// ---- walks -----------------------------------------------------------------------------------------------------------

// What the warps of a walk share beside the stages.  A wait that gives up ends all later ones of the CTA, and what is computed and stored
// from there on is NaN: whoever went on without what it waited for, and whose place it then took, finds the mark behind what it has read.
struct WalkShared {
    uint64_t full[4], empty[4], bar_a, bar_b, bar_c[2], bar_q, bar_y, bar_end; // copies; products; all of them
    uint64_t state[2], z_ready, u_ready, p_ready;             // the computing warps (of a half) to the one that issues
    uint64_t o_ready, o_taken;                                // the warps with the results to the one that issues
    float4 carry[4];                                          // of a stage's chunk (see Carry)
    unsigned slot;
    int gave_up, begun[4];                                    // begun: how often copies to a stage were begun
};
constexpr float kLost = __builtin_nanf("");
// Bounded by its polls, which sleep up to some microseconds each.  As few instructions as can be, for there are twenty of these waits in a
// walk's loop; who gives up leaves a mark, and the status is set at the kernel's end (see walk_end).
constexpr unsigned kWalkPolls = 1u << 20;
__device__ __forceinline__ void walk_wait(WalkShared *w, uint64_t *bar, unsigned parity)
{
    asm volatile("{\n .reg .pred p;\n .reg .u32 i, f;\n mov.u32 i, 0;\n"
                 "WALK_POLL_%=:\n mbarrier.try_wait.parity.shared::cta.b64 p, [%0], %1;\n @p bra WALK_DONE_%=;\n"
                 " ld.volatile.shared.u32 f, [%2];\n add.u32 i, i, 1;\n setp.lt.u32 p, i, %3;\n setp.eq.and.u32 p, f, 0, p;\n @p bra WALK_POLL_%=;\n"
                 " st.volatile.shared.u32 [%2], 1;\n"
                 "WALK_DONE_%=:\n}\n" ::"r"(smem_u32(bar)), "r"(parity), "r"(smem_u32(&w->gave_up)), "n"(kWalkPolls) : "memory");
}
__device__ __forceinline__ bool walk_given_up(const WalkShared *w) { return __builtin_expect(*(const volatile int *)&w->gave_up, 0); }
__device__ __forceinline__ void walk_late(WalkShared *w, bool late) { if (late) *(volatile int *)&w->gave_up = 1; }
__device__ __forceinline__ void walk_marks_init(WalkShared *w)
{
    mbar_init(&w->bar_end, 1);
    w->gave_up = w->begun[0] = w->begun[1] = w->begun[2] = w->begun[3] = 0;
    fence_mbar_init();
}
__device__ __forceinline__ void walk_last_wait(uint64_t *bar, unsigned parity)
{
#pragma unroll 1
    for (unsigned i = 0; i < kWalkPolls && !mbar_try_wait(bar, parity); ++i) { }
}
// The end of a CTA, by all its threads, `issuer` the warp that issued its products (-1: there are none).  Where a wait has given up no more
// copies were begun, and the CTA waits (bounded) for those under way and for its products, so that they end before the memory they
// work on is another CTA's.
__device__ __forceinline__ void walk_end(WalkShared *w, int stages, int *status, int warp, int issuer)
{
    __syncthreads();
    if (!w->gave_up) return;
    if (warp == issuer) {
        umma_commit(&w->bar_end);
        walk_last_wait(&w->bar_end, 0);
    }
    if (threadIdx.x == 0) {
        atomicExch(status, 1);
#pragma unroll 1
        for (int s = 0; s < stages; ++s)
            if (w->begun[s]) walk_last_wait(&w->full[s], (w->begun[s] - 1) & 1);
    }
    __syncthreads();
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory"); }
// Warps 0 .. 7 compute, warp 8 issues the products, warps 9 .. 11 fetch, warps 12 .. 15 take results away.  What is written into tensor
// memory is handed to warp 8 by barriers; what it gives back is seen by the products' barriers.
constexpr int kWalkThreads = 512, kFetchers = 96;
__device__ __forceinline__ void walk_init(WalkShared *w, int stages)
{
    for (int s = 0; s < stages; ++s) { mbar_init(&w->full[s], 2); mbar_init(&w->empty[s], 1); }
    mbar_init(&w->bar_a, 1); mbar_init(&w->bar_b, 1); mbar_init(&w->bar_c[0], 1); mbar_init(&w->bar_c[1], 1); mbar_init(&w->bar_q, 1); mbar_init(&w->bar_y, 1);
    mbar_init(&w->state[0], 4); mbar_init(&w->state[1], 4);
    mbar_init(&w->z_ready, 8); mbar_init(&w->u_ready, 8); mbar_init(&w->p_ready, 8); mbar_init(&w->o_ready, 4); mbar_init(&w->o_taken, 4);
    walk_marks_init(w);
}
__device__ __forceinline__ void walk_ready(uint64_t *bar, int lane)
{
    tmem_wait_st();
    tmem_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void fetchers_sync() { __syncwarp(); asm volatile("bar.sync 3, %0;\n" ::"n"(kFetchers) : "memory"); }
__device__ __forceinline__ void takers_sync() { asm volatile("bar.sync 2, 128;\n" ::: "memory"); }

__device__ __forceinline__ unsigned char *align_images(unsigned char *p) { return p + ((1024u - (smem_u32(p) & 1023u)) & 1023u); }

enum { WALK_RUN = 0, WALK_MAPS = 1 };
// A walk takes up to all the shared memory that a CTA can have, its images from the first byte of the dynamic part on, which starts on 1024
// bytes: it is declared so, and the static part, below that, is padded to it.
constexpr int kWalkStatic = 1024, kWalkBytes = 227 * 1024 - kWalkStatic;
static_assert(sizeof(WalkShared) <= kWalkStatic, "shared memory");

// ---- tensor copies -----------------------------------------------------------------------------------------------------

// Tiles of bf16 tensors whose rows start on 16 bytes come as tensor copies: rows behind a head's channels and tokens behind L arrive as
// zeros.  Others, and a chunk that ends before L, are fetched by threads (load_tile).
struct DeltaMaps { CUtensorMap k, q, v, more, out, outk; };        // v: values, or dy; more: values beside dy; out: y, dv or dq; outk: dk
__device__ __forceinline__ bool by_copy(const DeltaArgs &a, int nv, int t0) { return a.copies && (nv == kTok || t0 + nv == a.L); }

// ---- host ------------------------------------------------------------------------------------------------------------

// `v` as DeltaMaps has it; out, outk: results, of the keys' shape where there are two, of the values' where there is one (or none)
template <typename T> static bool delta_maps(DeltaMaps &m, const DeltaArgs &a, int rows, const void *v, const void *out, const void *outk)
{
    if (sizeof(T) != 2 || a.L % 8 || !tma_available()) return false;
    auto one = [&](CUtensorMap *map, const void *p, bool keys) {
        const int D = keys ? a.Dk : a.Dv;
        const unsigned long long dims[3] = {(unsigned long long)a.L, (unsigned long long)D, (unsigned long long)a.B * (keys ? a.Hk : a.H)},
                                 strides[2] = {2ull * a.L, 2ull * a.L * D};
        const unsigned box[3] = {(unsigned)kTok, (unsigned)rows, 1};
        return !p || tma_encode_3d(map, p, true, dims, strides, box, 128);
    };
    return one(&m.k, a.k, true) && one(&m.q, a.q, true) && one(&m.v, v, false) && one(&m.more, a.v, false) && one(&m.out, out, outk != nullptr) && one(&m.outk, outk, true);
}
struct DeltaSizes { size_t images, gates, maps, starts, dstates, dz, all; };          // bytes of the parts of a workspace, in this order
DeltaSizes delta_sizes(const DeltaArgs &a, int dtype, bool backward);
int launch_delta_prepare(DeltaArgs a, int dtype, cudaStream_t st);
int launch_delta_join(const DeltaArgs &a, const float *from, bool backward, cudaStream_t st);
int launch_delta_backward(const DeltaArgs &a, int dtype, cudaStream_t st);
int delta_backward_status();

// The walks and the gradients let the next kernel in at their end, prepare once its tensor memory is free, in front of the inverse.  Right
// behind the allocation, CTAs of the next came to the SMs that a walk of 96 heads leaves free and to no others (a training step on 6144 chunks
// 1312 us, so 1260).
template <auto FN, typename... M> static int launch_delta(const DeltaArgs &a, long long blocks, unsigned threads, int bytes, cudaStream_t st, const M &...maps)
{
    if (blocks > 0x7fffffffll) return kTooLarge;
    static PerDevice ready;
    if (bytes > 48 * 1024 - 4096 && !ready.once([&] { return cudaFuncSetAttribute(FN, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess ? 1 : -1; })) return kNoLaunch;
    launch_pdl(FN, dim3((unsigned)blocks), threads, bytes, st, a, maps...);
    return 0;
}

}  // namespace hn
