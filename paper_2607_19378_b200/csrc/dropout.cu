// Dropout from a counter-based generator: y = x * keep / (1 - p), the mask a function of (seed, step, site, element) that is
// worked out wherever it is needed and stored nowhere; the backward pass is the same call on dy.
//
// One pass over the data, 2 elements of traffic per element.  A thread takes octets of the flat tensor, one Philox call of
// ten rounds for eight elements (16 random bits each).
#include "entry.cuh"
#include "octet.cuh"
#include "philox.cuh"

namespace hn {

constexpr int kDropThreads = 256;

template <typename T> __global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T *x, T *y, long long n, DropArgs d)
{
    pdl_join();
    const DropKey key(d);
    const long long octets = (n + 7) >> 3;
    for (long long o = (long long)blockIdx.x * kDropThreads + threadIdx.x; o < octets; o += (long long)gridDim.x * kDropThreads) {
        const long long i = o << 3;
        Octet<T> raw;
        raw.ld(x, i, n);
        const unsigned keep = key.keep(o);
        float f[8];
        raw.get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = keep >> e & 1 ? f[e] * d.scale : 0.f;       // (dropped: zero, whatever was there)
        st_octet(y, i, 0, n - i < 8 ? (int)(n - i) : 8, f);
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
    const long long octets = (n + 7) / 8, blocks = (octets + kDropThreads - 1) / kDropThreads;
    const dim3 grid((unsigned)(blocks < kSms * 8 ? blocks : kSms * 8));
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == HYENAND_F32) launch_pdl(dropout_kernel<float>, grid, kDropThreads, 0, st, (const float *)x, (float *)y, n, d);
    else launch_pdl(dropout_kernel<bf16>, grid, kDropThreads, 0, st, (const bf16 *)x, (bf16 *)y, n, d);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? HYENAND_OK : fail(HYENAND_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}
