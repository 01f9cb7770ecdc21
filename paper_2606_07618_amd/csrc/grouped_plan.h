// Which kernel a product of rows sorted by group runs.  Arithmetic on sizes alone, without the device's headers, so that a
// host compiler takes it too.
#pragma once

#include "product_plan.h"

namespace grouped_plan {

using product_plan::ceil_div;

constexpr int kLargeTile = 256, kSmallTile = 128;        // rows, and as many outputs
constexpr int kLargeThreads = 512, kSmallThreads = 256;
constexpr int kFewThreads = 256;                         // few rows: a four of waves
constexpr int kFewFours = 2;                             // of them along the contraction, of 16 rows where workgroups are few
constexpr int kUnits = 32, kXcds = 8;                    // compute units of an XCD

struct GroupedPlan { int height, width, threads; };

// By the rows that a group has on average (how many each has is known on the device alone; every kernel takes
// any number).  Few rows: 16 or 32 of a group at a time, and 128 weight rows a workgroup, or 64 where those would be few.  Measured
// with 12 to 32 rows a group, 8 to 128 groups, contractions of 1024 to 14336: 0.34 to 0.99 of the tiles' time.  33 to 64 rows a
// group go that way below 512 tiles.  With 256 to 480 tiles and groups as uneven as a router's (shares of 1 / (i + 1)^0.6 and 1.2) that
// took 0.53 to 0.99 of the tiles' time in 38 of 40 cases (60 groups of 36 rows, [1024, 4096]: 56 to 66 us, 70 to 93 in tiles); groups that
// are all alike are faster in tiles from 320 on (60 of 48 rows: 66 and 49), which their average does not tell.  From 512 on: 128
// groups of 50 rows, [1536, 4096], 215 us, 171 in tiles.  The largest tile where groups fill it more than half and three quarters
// of the compute units have one (128 of 200 rows, [1536, 4096]: 350 us, 457 in the smaller one).
inline GroupedPlan plan_grouped(int64_t rows, int64_t experts, int64_t outer, bool turned) {
    const int64_t active = rows < experts ? rows : experts, each = active ? ceil_div(rows, active) : 0;
    if (!turned && (each <= 32 || (each <= 64 && active * ceil_div(outer, kSmallTile) < 512))) {
        const int height = each <= 16 ? 16 : 32;
        const int64_t tiles = active * ceil_div(each, height);
        const int width = tiles * ceil_div(outer, 128) >= 512 ? 128 : 64;
        return {height, width, kFewThreads * (height == 16 && width == 64 ? kFewFours : 1)};
    }
    if (each > 128 && active * ceil_div(each, kLargeTile) * ceil_div(outer, kLargeTile) >= 192) return {kLargeTile, kLargeTile, kLargeThreads};
    return {kSmallTile, kSmallTile, kSmallThreads};
}

// Workgroups: for the row tiles that there may be, each XCD as many, and one at least that finds rows of no group to clear;
// and for the parts that its last tiles are cut into.
inline int64_t most_groups_of(int64_t rows, int64_t experts, int64_t outer, const GroupedPlan& plan) {
    const int64_t tiles = rows / plan.height + (rows < experts ? rows : experts);
    const int64_t more = plan.height == kLargeTile ? kUnits : 1;
    return (ceil_div(tiles * ceil_div(outer, plan.width), kXcds) + more) * kXcds;
}

}  // namespace grouped_plan
