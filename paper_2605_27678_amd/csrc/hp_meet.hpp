// How the waves of a workgroup meet over tiles in LDS.  Plain arithmetic that the kernels and the CPU's tests share.
#pragma once

namespace hp {

// Loads that a wave of 64 lanes makes of `pieces`, one a lane, in rounds of `threads` lanes; pieces are whole waves' loads.
// Where the last round is not a whole one, later waves make one less: what a wave waits for goes by its own.
constexpr int loads_of_wave(int pieces, int threads, int wave) { return pieces / threads + (64 * wave < pieces % threads ? 1 : 0); }

// Loads of a wave that may still be under way when a tile is read, if it makes `each` a tile and has asked for `behind`
// tiles after that one (loads end in the order in which they were made).
constexpr int under_way(int each, int behind) { return behind > 0 ? each * behind : 0; }

// A flag that any wave may have set, read by all of them alike: `meet` is the workgroup's barrier.  The second one keeps a
// wave that goes on (and may clear the flag for what comes next) from those that have not read it yet.
template <class Meet> constexpr int read_together(const int *flag, const Meet &meet) {
    meet();
    const int set = *flag;
    meet();
    return set;
}

}  // namespace hp
