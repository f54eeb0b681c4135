// The turns that the converter warps of the score-cache kernel take at a unit's tiles (page scales over an 8-bit cache): what a warp
// waits for, when it expands and when it arrives.  Apart from the kernel, so that a host model can run these very steps.
//
// Two teams of two warps expand every other tile, so that one team's loads and conversions run under the other's waits and fences.
// A wait on an mbarrier's parity tells only its last two phases apart.
//  - Both teams therefore wait for every tile's stage and slot: with an odd number of either, a team's next turn at one of them
//    comes two phases on, and it must have seen the one between.
//  - And both arrive for every tile: were a stage free, or a slot full, once its own team has expanded it, TMA or the tensor cores could
//    complete the next phase there before a late warp of the other team has looked at this one, and that warp would wait
//    for a phase that cannot come without it.  The team whose turn it is not arrives as soon as its waits are over.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define SPEC_TURNS __device__ __forceinline__
#else
#define SPEC_TURNS inline
#endif

namespace spec {

constexpr int kConverterWarps = 4;
constexpr int kConverterArrivals = kConverterWarps;  // per phase of raw_empty and slot_full

struct ConverterTurns {
    uint32_t r = 0, rph = 0;    // raw stage of the next tile, its phase
    uint32_t sl = 0, sph = 0;   // operand slot, likewise
    uint32_t g = 0;             // tiles so far, of both teams
};

// wait(stage, its phase, slot, its phase): false if the wait was abandoned.  arrive(stage, slot): on raw_empty and slot_full.
template <class Wait, class Expand, class Arrive>
SPEC_TURNS bool converter_tiles(ConverterTurns& t, int n_tiles, uint32_t team, uint32_t n_raw, uint32_t n_slots, const Wait& wait,
                                const Expand& expand, const Arrive& arrive)
{
    for (int c = 0; c < n_tiles; ++c, ++t.g) {
        if (!wait(t.r, t.rph, t.sl, t.sph ^ 1)) return false;
        if ((t.g & 1) == team) expand(t.r, t.sl);
        arrive(t.r, t.sl);
        if (++t.r == n_raw) {
            t.r = 0;
            t.rph ^= 1;
        }
        if (++t.sl == n_slots) {
            t.sl = 0;
            t.sph ^= 1;
        }
    }
    return true;
}

}  // namespace spec
