// What one launch holds: HIP numbers its threads in 32 bits.
#pragma once

#include <stdint.h>

// Workgroups of `threads` that one launch takes, and whether it takes `groups` of them.
constexpr int64_t most_groups(int threads) { return (int64_t)0xFFFFFFFF / threads; }
constexpr bool launchable(int64_t groups, int threads) { return groups <= most_groups(threads); }
