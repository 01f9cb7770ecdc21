// Which kernel a matrix product runs: its tile, its parts, the forms for few rows.  Arithmetic on sizes alone, without the
// device's headers, so that a host compiler takes it too.
#pragma once

#include <stdint.h>

#include "launch_limit.h"

namespace product_plan {

inline int64_t up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Microscaled operands' scales as the rows lie (kMx, rows of whole words), or laid out step by step (kMxLaid).  kInt8:
// 8-bit integers, sums in 32 bits, exact, and a scale for each row of either operand.
enum Kind { kBf16, kMx, kMxLaid, kInt8 };
template <Kind KIND> constexpr bool kMicroscaled = KIND == kMx || KIND == kMxLaid;

// What happens to the sums.
enum Out {
    kSums,        // scale * sum, as bfloat16 or binary32
    kPartial,     // the sum of this part of the contraction, binary32, for a later reduction
    kGate,        // B is two matrices: silu(sum of the first) * sum of the second, and both sums where asked for;
                  // a tile's outer indexes of B are taken half from each, so that an output's two sums meet in one lane
    kGatePartial, // both sums of this part of the contraction, [part][2][m][n] in binary32
    kTwoRows,     // rows below `half_rows` to the first output, those from there on to the second
    kAdded        // the sum on top of what the binary32 output holds
};

// ---- the tile and the split of a product --------------------------------------------------------
// Four tiles, from the one that moves least through LDS for what it computes to the one that gives the most
// workgroups; and the contraction may be split over workgroups, whose sums a second kernel adds.  The rule takes the
// least estimated time, from what each tile took on this card with contractions of 128 to 4096 values: with a workgroup
// on few of the 256 compute units `start` + steps * `alone` microseconds, and with many workgroups `fixed` (filling
// the pipeline, storing the tile) + steps * `among` for each 256 of them.
//   measured, bfloat16, contraction 384: [8192, 8192] outputs 70 us with the largest tile, 86, 118, 159 with the
//   next; [256, 2048] outputs 16.1, 9.8, 7.0, 5.5 us.
struct TileCost { int m, n; float start, alone, fixed, among; };
constexpr int kTiles = 4, kMostParts = 16;
constexpr float kLaunchUs = 2.0f;
constexpr float kJoinUs = 6.0f, kJoinBytesUs = 8e6f;     // a second launch; bytes a microsecond
constexpr float kSmaller = 0.93f;                        // a smaller tile reads more: taken where it is clearly faster
constexpr float kLayUs = 6.0f;                           // a launch that lays scales out

template <Kind KIND>
inline const TileCost* tile_costs() {
    static constexpr TileCost mx[kTiles] = {{256, 256, 7.0f, 1.5f, 9.0f, 1.7f}, {128, 128, 6.3f, 1.1f, 1.9f, 0.75f},
                                            {64, 128, 5.1f, 0.64f, 1.4f, 0.48f}, {64, 64, 4.4f, 0.40f, 1.3f, 0.31f}};
    static constexpr TileCost bf16[kTiles] = {{256, 256, 9.8f, 1.05f, 8.5f, 1.54f}, {128, 128, 5.1f, 0.77f, 2.5f, 0.51f},
                                              {64, 128, 4.7f, 0.38f, 1.7f, 0.34f}, {64, 64, 3.7f, 0.31f, 1.3f, 0.23f}};
    // kInt8: a step has as many bytes and takes as long in the matrix instructions as bfloat16's.  (No estimate counts how fast
    // operands come from memory: [48, 8192] x [28672, 8192] in integers is estimated at 29 us and takes 56.)
    return kMicroscaled<KIND> ? mx : bf16;
}

// Fragments of a wave's rows of A and of B.
constexpr int kFragments[kTiles][2] = {{8, 4}, {4, 4}, {2, 4}, {2, 2}};

struct Plan { int tile, parts; float us; };

// Values of a step of the contraction, and outer indexes of B for an output.
template <Kind KIND> constexpr int kStepValues = kMicroscaled<KIND> ? 256 : KIND == kInt8 ? 128 : 64;
template <Out OUT> constexpr int kHalf = OUT == kGate ? 2 : 1;

// Estimated microseconds with tile t and the contraction in `parts`.  Up to a workgroup a compute unit, what they take
// of each other grows with their number ([1024, 4096] x [4096, 4096], where the largest tile in four parts makes 256
// workgroups, estimated as if each were alone: 66 us; with a smaller tile, taken since, 57).
template <Kind KIND, Out OUT>
float product_us(int t, int parts, int64_t m, int64_t n, int64_t inner) {
    const TileCost& cost = tile_costs<KIND>()[t];
    const float tiles = (float)ceil_div(m, cost.m) * (float)ceil_div(n * kHalf<OUT>, cost.n);
    const float load = tiles * parts / 256.0f, own = (float)ceil_div(ceil_div(inner, kStepValues<KIND>), parts);
    const float share = load <= 1.0f && cost.among > cost.alone ? (cost.among - cost.alone) * load : 0.0f;
    const float few = cost.start + own * (cost.alone + share);
    const float many = load > 1.0f ? kLaunchUs + (float)(int64_t)(load + 0.999f) * (cost.fixed + own * cost.among) : 0.0f;
    float us = few > many ? few : many;
    if (kMicroscaled<KIND> && t == 0) us += kLayUs;
    // kInt8: a step's values are twice as many, so that parts are short and cost more than their sums' bytes; these are counted
    // twice.  That changes one plan in forty (of 5 to 8192 rows, 64 to 28672 outputs, 64 to 14336 values); 54 such products
    // timed both ways take 4 % less on average: 14 % where it takes fewer parts of a split ([777, 14336] x [1001, 14336]: 33 us in
    // two parts of the third tile, 36 in eight of the second), but 4 % more where it takes a whole product in place of a split.
    constexpr int kBytes = KIND == kInt8 ? 16 : 8;
    if (parts > 1) us += kJoinUs + (float)m * (float)n * (float)(kBytes * kHalf<OUT> * parts) / kJoinBytesUs;
    return us;
}

template <Kind KIND, Out OUT>
Plan plan_product(int64_t m, int64_t n, int64_t inner) {
    const int64_t steps = ceil_div(inner, kStepValues<KIND>);
    Plan best = {0, 1, 3e38f};
    for (int t = 0; t < kTiles; ++t) {
        if (OUT == kGate && tile_costs<KIND>()[t].n < 128) continue;   // a wave holds both products of 32 columns
        for (int parts = 1; parts <= kMostParts && (parts == 1 || steps / parts >= 8); parts *= 2) {
            const float us = product_us<KIND, OUT>(t, parts, m, n, inner);
            if (us < best.us * (t > best.tile ? kSmaller : 1.0f)) best = {t, parts, us};
        }
    }
    return best;
}

constexpr int kTileThreads[kTiles] = {512, 256, 256, 256}, kJoinThreads = 256;

// Whether the launches of a product fit, all of them: asked before the first one of a call.
template <Kind KIND, Out OUT = kSums>
bool product_launchable(int64_t m, int64_t n, int64_t inner) {
    const Plan p = plan_product<KIND, OUT>(m, n, inner);
    const TileCost& tile = tile_costs<KIND>()[p.tile];
    const int64_t tiles = ceil_div(m, tile.m) * ceil_div(n * kHalf<OUT>, tile.n);
    return launchable(tiles * p.parts, kTileThreads[p.tile]) &&
           (p.parts == 1 || launchable(ceil_div(m * n, kJoinThreads), kJoinThreads));
}

// Bytes of the parts' sums, 0 where the product is not split.
template <Kind KIND, Out OUT = kSums>
int64_t parts_bytes(int64_t m, int64_t n, int64_t inner) {
    const Plan p = plan_product<KIND, OUT>(m, n, inner);
    return p.parts > 1 ? up(p.parts * m * n * (OUT == kGate ? 8 : 4), 256) : 0;
}

// ---- products with few rows -----------------------------------------------------------------------

constexpr int kDotRows = 4;                      // dot products: this many rows of activations

// Up to this many rows the weights are expanded in registers, on their way into the matrix instructions, once for each
// 128 rows; beyond, once and for all, and multiplied as bfloat16 tiles.  Measured, expanded in registers and beforehand:
// [14336, 4096] 16 rows 18 and 50 us, 128 rows 31 and 56, 512 rows 81 and 89, 640 rows 118 and 106;
// [28672, 8192] 512 rows 302 and 307, 1024 rows 525 and 468.
constexpr int64_t kStreamRows = 512;

constexpr int kStreamRowsN = 128;                // weight rows of a workgroup
constexpr int kWavesK = 2;                       // waves along the contraction, a half each
constexpr int kGroup = 256;                      // values of a weight row whose scales are loaded together

// 32 activation rows each, of a workgroup.
inline int stream_rows_of(int64_t m) { return m <= 32 ? 1 : m <= 64 ? 2 : 4; }
inline int stream_tiles_m(int64_t m) { return (int)((m + 127) / 128); }

// Values of a part: halves of whole groups.
inline int stream_part_values(int64_t k, int parts) {
    constexpr int64_t kUnit = kGroup * kWavesK;
    return (int)(((k + parts - 1) / parts + kUnit - 1) / kUnit * kUnit);
}

// A workgroup takes a compute unit's LDS, so 256 of them work at a time, and a value of the contraction takes each 5.3, 7
// or 10 ns (32, 64 or 128 rows).  Parts of it, of at least 1024 values, where rounds and the parts' sums then take less
// ([384, 14336] x [4096, 14336]: 102 us in three parts of 288 workgroups together, 79 in two of 192).
inline int stream_parts(int64_t m, int64_t n, int64_t k) {
    const int64_t groups = (n + kStreamRowsN - 1) / kStreamRowsN * stream_tiles_m(m);
    const float us = (stream_rows_of(m) == 1 ? 0.0053f : stream_rows_of(m) == 2 ? 0.007f : 0.01f);
    int best = 1;
    float least = 3e38f;
    for (int p = 1; p <= 16 && (p == 1 || k / p >= 1024); ++p) {
        const float took = (float)((groups * p + 255) / 256) * (float)stream_part_values(k, p) * us +
                           (p > 1 ? 6.0f + (float)m * (float)n * (float)(8 * p) / 4e6f : 0.0f);
        if (took < least) least = took, best = p;
    }
    return best;
}

constexpr int kThinRows = 16;                    // microscaled products without tiles: at most

// Estimated microseconds: one row, [4096, 4096] 5.2, [4096, 14336] 10.9, [28672, 8192] 36; 16 rows 6.7, 16.5 and 55.
inline float thin_us(int64_t m, int64_t n, int64_t k) { return 2.0f + (float)n * (float)k * (1.6e-7f + 0.7e-8f * (float)m); }

// Few rows: the kernel for them where tiles, which must be many or be split to keep the chip busy, would take longer.
inline bool thin(int64_t m, int64_t n, int64_t blocks) {
    return m <= kThinRows && thin_us(m, n, blocks * 32) < plan_product<kMx, kSums>(m, n, blocks * 32).us;
}

// The largest tile takes its scales laid out, and so do the others where rows of scales are no whole words.
inline bool lays_scales(int64_t m, int64_t n, int64_t blocks) {
    return blocks % 4 != 0 || plan_product<kMx, kSums>(m, n, blocks * 32).tile == 0;
}

}  // namespace product_plan
