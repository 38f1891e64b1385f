// How the warps of an epilogue walk over their block's tiles, alternating between two accumulators.  Ordinary C++ on a
// host compiler, so that what happens when a warp gives up can be run there.
#pragma once

#ifdef __CUDACC__
#define CMPQ_WALK __device__ __forceinline__
#else
#define CMPQ_WALK inline
#endif

namespace cmpq {

// Every warp calls this with the same tiles.  `meet(tile, acc)` ends in a barrier of all these warps, so each of them goes
// through it for every tile, also after it has given up; `ready(acc, parity)` waits, with a limit, for the accumulator;
// `take(tile, acc)` reads it and hands it back.  A warp that gave up takes nothing any more.
template <class Meet, class Ready, class Take>
CMPQ_WALK void walk_tiles(int first, int tiles, int step, Meet meet, Ready ready, Take take) {
    int acc = 0, parity = 0;
    bool ok = true;
    for (int tile = first; tile < tiles; tile += step) {
        meet(tile, acc);
        ok = ok && ready(acc, parity);
        if (ok) take(tile, acc);
        acc ^= 1;
        if (acc == 0) parity ^= 1;
    }
}

}  // namespace cmpq
