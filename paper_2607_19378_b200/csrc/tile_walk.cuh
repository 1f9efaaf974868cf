// How a CTA or cluster walks over the tiles of a batch (internal; host code can include it).
#pragma once

#ifdef __CUDACC__
#define HN_HD __host__ __device__ __forceinline__
#else
#define HN_HD inline
#endif

namespace hn {

// Every `step`-th tile, as batch entry and tile of it, without a division per tile.  A walk goes up to two steps beyond the last
// entry, which may be the 2^31 - 1st: entries are counted without a sign.
struct TileWalk {
    unsigned b;                                              // entry
    int r;                                                   // tile of the entry
    unsigned step_b;
    int step_r, per;
    HN_HD TileWalk(long long first, long long step, int tiles_b) : b((unsigned)(first / tiles_b)), r((int)(first % tiles_b)),
        step_b((unsigned)(step / tiles_b)), step_r((int)(step % tiles_b)), per(tiles_b) {}
    HN_HD bool inside(int entries) const { return b < (unsigned)entries; }
    HN_HD void next()
    {
        b += step_b; r += step_r;
        if (r >= per) { r -= per; ++b; }
    }
};

}  // namespace hn
