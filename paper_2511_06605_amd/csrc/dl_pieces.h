// How long pieces of a key axis are where lengths alone say it (dl_chunk.hip); whole numbers, the same on the host.
#pragma once

#include <stdint.h>

// No sequence has so many steps (2^30 tokens, 64 a step at least): pieces of this size cut none.
constexpr uint32_t DL_UNCUT = 1u << 26;

// Steps of a piece, where all tiles have `all` steps together and pieces of sequences that are cut may be no more than most_cut >= 2.
// Those have more steps than a piece, so fewer pieces than 2 steps / size each, and 2 all / size <= most_cut in all.  The quotient may have more
// than 32 bits (131 073 tiles of 2^30 tokens each and 1024 pieces: 2^32 + 2^15): from DL_UNCUT on it says the same.
constexpr uint32_t dl_piece_steps(uint64_t all, uint32_t most_cut)
{
    const uint64_t half = most_cut / 2u, size = (all + half - 1u) / half;
    return size > DL_UNCUT ? DL_UNCUT : size ? (uint32_t)size : 1u;
}
