// How the positions that a tile's rows see are split into parts (see find_unit): plain arithmetic, the same for every compiler.
#pragma once

#include <stdint.h>

namespace hbp {

constexpr int kStep = 32;   // positions that a matrix instruction takes at once; parts begin at multiples of it

// Positions of a part, a multiple of kStep, of `total` tiles times positions in all: about total / places, at most `enough`; but not less than `least`, nor than total / aim, which bounds how many parts there are
// whatever `enough` says.  (No text has 2^31 - 65536 positions: the longest parts hold any.)
constexpr int32_t part_length(double total, int32_t places, int32_t aim, int32_t enough, int32_t least)
{
    const double by_places = total / places, by_aim = total / aim;
    double share = by_places < enough ? by_places : enough;
    if (share < by_aim) share = by_aim;
    if (share < least) share = least;
    constexpr double kMost = 2147483616.0;   // 2^31 - kStep
    if (share > kMost) share = kMost;
    int32_t length = (int32_t)share;
    length += length < share;
    return (int32_t)(((uint32_t)length + kStep - 1) / kStep * kStep);
}

// Parts of a tile that sees up to `span` positions; up to `whole` are not split.
constexpr int32_t part_count(int32_t span, int32_t length, int32_t whole)
{
    return span <= whole ? 1 : (int32_t)(((uint32_t)span + (uint32_t)length - 1) / (uint32_t)length);
}

}  // namespace hbp
