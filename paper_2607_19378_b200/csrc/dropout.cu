// Dropout from a counter-based generator: y = x * keep / (1 - p), the mask a function of (seed, step, site, element) that is
// worked out wherever it is needed and stored nowhere; the backward pass is the same call on dy.
//
// One pass over the data.  A thread takes four octets of bf16 or two of fp32, one Philox call of ten rounds for eight elements (16
// random bits each): 15 instructions an element.  50 M elements behind a cold L2: fp32 64 us (0.96 of the measured bandwidth), bf16 46 us
// (0.66), in calls that follow each other 40 (0.75): the generator's integer instructions take the ALU to 55 %, and the warps wait for
// their loads and for that pipe in turn.
// Threads that walk over several such pieces: 84 and 48 us.
#include "entry.cuh"
#include "octet.cuh"
#include "pair.cuh"
#include "philox.cuh"

namespace hn {

constexpr int kDropThreads = 256, kDropCtas = 4;             // an SM holds

template <typename T> __global__ void __launch_bounds__(kDropThreads, kDropCtas) dropout_kernel(const T *x, T *y, long long n, DropArgs d)
{
    constexpr int U = 8 / (int)sizeof(T);                    // octets of a thread on their way at once
    pdl_join();
    const DropKey key(d);
    const long long octets = (n + 7) >> 3, stride = kDropThreads, o = (long long)blockIdx.x * U * kDropThreads + threadIdx.x;
    if (o < octets) {
        Octet<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (o + u * stride < octets) raw[u].ld(x, (o + u * stride) << 3, n);
        uint4 w[U];
        key.words(o, stride, w);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long at = o + u * stride, i = at << 3;
            if (at >= octets) break;
            float f[8];
            raw[u].get(f);
            const unsigned v[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {                    // (dropped: zero, whatever was there)
                const f2 k = mul2(make2(f[2 * j], f[2 * j + 1]), pair(d.scale));
                f[2 * j] = key.low(v[j]) ? k.x : 0.f;
                f[2 * j + 1] = key.high(v[j]) ? k.y : 0.f;
            }
            st_octet(y, i, 0, n - i < 8 ? (int)(n - i) : 8, f);
        }
    }
}

// false: p is not a probability below 1
bool drop_args(float p, const long long *rng, int site, DropArgs *d)
{
    if (!(p >= 0.f && p < 1.f)) return false;
    unsigned t = (unsigned)((double)p * 65536.0 + 0.5);
    if (t > 65535) t = 65535;
    d->rng = rng; d->site = (unsigned)site; d->threshold = t; d->scale = (float)(65536.0 / (65536 - t));
    return true;
}

}  // namespace hn

using namespace hn;

extern "C" int hyenand_dropout(long long n, int dtype, const void *x, float p, const long long *rng, int site, void *y, void *cuda_stream)
{
    clear_error();
    if (n < 1) return fail(HYENAND_ERR_INVALID_ARG, "n must be >= 1");
    if (dtype != HYENAND_F32 && dtype != HYENAND_BF16) return fail(HYENAND_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (!x || !y || !rng) return fail(HYENAND_ERR_INVALID_ARG, "x, rng, y must be non-NULL");
    DropArgs d;
    if (!drop_args(p, rng, site, &d)) return fail(HYENAND_ERR_INVALID_ARG, "p must be in [0, 1)");
    CallTensors c;
    c.in("x", x, (size_t)n * elsize(dtype));
    c.in("rng", rng, 2 * sizeof(long long));
    c.out("y", y, (size_t)n * elsize(dtype), 16, x);
    if (int e = c.check()) return e;
    c.register_ranges();
    const long long octets = (n + 7) / 8, each = kDropThreads * (8 / (long long)elsize(dtype)), blocks = (octets + each - 1) / each;
    if (blocks > 0x7fffffffll) return fail(HYENAND_ERR_UNSUPPORTED, "n is too large for one launch");
    const dim3 grid((unsigned)blocks);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == HYENAND_F32) launch_pdl(dropout_kernel<float>, grid, kDropThreads, 0, st, (const float *)x, (float *)y, n, d);
    else launch_pdl(dropout_kernel<bf16>, grid, kDropThreads, 0, st, (const bf16 *)x, (bf16 *)y, n, d);
    return finish(0);
}
