// What the C entry points share: the calling thread's error message, the address ranges of the checked build, and the rule on
// overlapping arguments (internal).
#pragma once
#include <stdint.h>

#include <mutex>

#include "../../include/hyenand.h"
#include "common.cuh"

namespace hn {

int fail(int code, const char *fmt, ...);            // records the message for hyenand_last_error, returns the code
void clear_error();                                  // at the head of every entry point

static inline size_t elsize(int dtype) { return dtype == HYENAND_F32 ? 4 : 2; }

// What became of a call's launches; `launched` below 0: one was not made (kTooLarge, or the runtime's error says why).  The error is
// taken with it: left behind, it would be the next call's, whose kernel is on its way.
constexpr int kNoLaunch = -1, kTooLarge = -2;
static inline int finish(int launched)
{
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fail(HYENAND_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    if (launched == kTooLarge) return fail(HYENAND_ERR_UNSUPPORTED, "kernel grid too large for one launch");
    return launched < 0 ? fail(HYENAND_ERR_CUDA, "kernel launch failed: the device holds no such CTA or cluster") : HYENAND_OK;
}

// What a launch works out once per device (a kernel's limits, how many of its CTAs run at once), whichever thread comes first.
struct PerDevice {
    std::mutex lock;
    int value[64] = {0};                             // 0: not worked out yet
    template <typename F> int get(F f)               // f() > 0, or -1: it failed, and is tried again at the next call
    {
        int dev = 0;
        cudaGetDevice(&dev);
        std::lock_guard<std::mutex> hold(lock);
        int &v = value[dev & 63];
        if (v <= 0) v = f();
        return v;
    }
    template <typename F> bool once(F f) { return get(f) > 0; }
};

// Checked build: the address ranges a call may touch (the caller's tensors, the device allocations of the objects
// involved), handed to every translation unit before the call's kernels are enqueued.
struct DbgScope {
#ifdef HYENAND_DEBUG
    DbgRanges r;
    DbgScope() { r.n = 0; }
    void add(const void *ptr, size_t bytes)
    {
        if (ptr && bytes && r.n < kDbgRanges) { r.lo[r.n] = (unsigned long long)ptr; r.hi[r.n] = r.lo[r.n] + bytes; ++r.n; }
    }
    void add(const GuardedAllocs &g)
    {
        for (int i = 0; i < g.n; ++i) add(g.recs[i].base + kGuardBytes, g.recs[i].bytes);
    }
    void commit()
    {
        cudaDeviceSynchronize();               // kernels of earlier calls still compare against the previous list
        dbg_set_ranges(r);
    }
#else
    void add(const void *, size_t) {}
    void add(const GuardedAllocs &) {}
    void commit() {}
#endif
};

// The tensors of one call.  Inputs may overlap one another, an output may overlap nothing else (`with`: the one input it may be
// the same buffer as, where every element is read before the thread that replaces it does so).
struct CallTensors {
    struct One { const void *ptr; size_t bytes; const char *name; int align; bool out; const void *with; };
    One t[24];
    int n = 0;
    void in(const char *name, const void *ptr, size_t bytes, int align = 16) { if (ptr && bytes) t[n++] = {ptr, bytes, name, align, false, nullptr}; }
    void out(const char *name, const void *ptr, size_t bytes, int align = 16, const void *with = nullptr)
    {
        if (ptr && bytes) t[n++] = {ptr, bytes, name, align, true, with};
    }
    int check() const
    {
        for (int i = 0; i < n; ++i)
            if ((uintptr_t)t[i].ptr % t[i].align) return fail(HYENAND_ERR_INVALID_ARG, "%s is not %d-byte aligned", t[i].name, t[i].align);
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j) {
                if (i == j || !t[i].out) continue;
                if (!t[j].out && t[i].with == t[i].ptr && t[j].ptr == t[i].ptr && t[j].bytes == t[i].bytes) continue;
                const char *a = (const char *)t[i].ptr, *b = (const char *)t[j].ptr;
                if (a < b + t[j].bytes && b < a + t[i].bytes) return fail(HYENAND_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, t[j].name);
            }
        return HYENAND_OK;
    }
    void register_ranges() const
    {
        DbgScope d;
        for (int i = 0; i < n; ++i) d.add(t[i].ptr, t[i].bytes);
        d.commit();
    }
};

}  // namespace hn
