// Host side of the matrix products: the checks that every product shares, the plan of its tiles, and
// the kernels that bring an operand into the form the tiles read.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "launch_limit.h"
#include "nvfp4ss.h"
#include "tile_product.h"

namespace product_host {

using namespace tile_product;

// A tile's loads take 32-bit offsets from its first row: 256 rows of this many bfloat16 values stay
// below the 2 GiB window.
constexpr int64_t kMaxWidth = (int64_t)1 << 20, kMaxLd = (int64_t)1 << 21;
constexpr int64_t kMaxRows = (int64_t)1 << 36;      // workspace sizes stay within 63 bits

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
inline int64_t up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_dims(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0 || m > kMaxRows || n > kMaxWidth || k > kMaxWidth) return NVFP4_ERR_SHAPE;
    return NVFP4_OK;
}

inline int launched() { return hipGetLastError() == hipSuccess ? NVFP4_OK : NVFP4_ERR_HIP; }

// Rows of `width` values as the tiles read them: 16-byte chunks, zeros past the width.
inline bool needs_pack(int64_t width, int64_t ld) { return width % 8 != 0 || ld % 8 != 0; }
inline int64_t packed_ld(int64_t width) { return up(width, 8); }

// Sections of a caller's workspace, 256-byte aligned.  With a null base it only measures.
struct Carver {
    char* base;
    int64_t at = 0;
    void* take(int64_t bytes) {
        void* p = base ? base + at : nullptr;
        at += up(bytes, 256);
        return p;
    }
};

int pack_bf16_rows(const void* src, int64_t rows, int64_t width, int64_t ld, void* dst, hipStream_t stream);

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
    return KIND != kBf16 ? mx : bf16;
}

// Fragments of a wave's rows of A and of B.
constexpr int kFragments[kTiles][2] = {{8, 4}, {4, 4}, {2, 4}, {2, 2}};

struct Plan { int tile, parts; float us; };

template <Kind KIND, Out OUT>
Plan plan_product(int64_t m, int64_t n, int64_t inner) {
    constexpr int kStepValues = KIND != kBf16 ? 256 : 64, kHalf = OUT == kGate ? 2 : 1;
    const int64_t steps = ceil_div(inner, kStepValues);
    const TileCost* costs = tile_costs<KIND>();
    Plan best = {0, 1, 3e38f};
    for (int t = 0; t < kTiles; ++t) {
        if (OUT == kGate && costs[t].n < 128) continue;        // a wave holds both products of 32 columns
        const float tiles = (float)ceil_div(m, costs[t].m) * (float)ceil_div(n * kHalf, costs[t].n);
        for (int parts = 1; parts <= kMostParts && (parts == 1 || steps / parts >= 8); parts *= 2) {
            const float load = tiles * parts / 256.0f, own = (float)ceil_div(steps, parts);
            const float share = load < 1.0f && costs[t].among > costs[t].alone ? (costs[t].among - costs[t].alone) * load : 0.0f;
            const float few = costs[t].start + own * (costs[t].alone + share);
            const float many = load > 1.0f ? kLaunchUs + (float)(int64_t)(load + 0.999f) * (costs[t].fixed + own * costs[t].among) : 0.0f;
            float us = few > many ? few : many;
            if (KIND != kBf16 && t == 0) us += kLayUs;
            if (parts > 1) us += kJoinUs + (float)m * (float)n * (float)(8 * kHalf * parts) / kJoinBytesUs;
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
    const int64_t tiles = ceil_div(m, tile.m) * ceil_div(n * (OUT == kGate ? 2 : 1), tile.n);
    return launchable(tiles * p.parts, kTileThreads[p.tile]) &&
           (p.parts == 1 || launchable(ceil_div(m * n, kJoinThreads), kJoinThreads));
}

// Bytes of the parts' sums, 0 where the product is not split.
template <Kind KIND, Out OUT = kSums>
int64_t parts_bytes(int64_t m, int64_t n, int64_t inner) {
    const Plan p = plan_product<KIND, OUT>(m, n, inner);
    return p.parts > 1 ? up(p.parts * m * n * (OUT == kGate ? 8 : 4), 256) : 0;
}

// Fills in the tiles and steps of p and launches; p's operands, outer indexes and outputs are set.
template <Kind KIND, Out OUT, class T>
int launch_tiles(Args p, hipStream_t stream) {
    constexpr int kStepValues = KIND != kBf16 ? 256 : 64;
    p.steps = ceil_div(p.inner, kStepValues);
    p.tiles_m = ceil_div(p.m, T::M);
    p.tiles_n = ceil_div(p.n, OUT == kGate || OUT == kGatePartial ? T::N / 2 : T::N);
    p.split_steps = ceil_div(p.steps, p.parts);
    if (!launchable(p.tiles_m * p.tiles_n * p.parts, T::kThreads)) return NVFP4_ERR_SHAPE;
    if (p.tiles_m * p.tiles_n == 0) return NVFP4_OK;
    hipLaunchKernelGGL((product_kernel<KIND, OUT, T>), dim3((unsigned)(p.tiles_m * p.tiles_n * p.parts)),
                       dim3(T::kThreads), 0, stream, p);
    return launched();
}

using Tile0 = Tile<256, 256, 2, 4>;
using Tile1 = Tile<128, 128, 2, 2>;
using Tile2 = Tile<64, 128, 2, 2, 3>;
using Tile3 = Tile<64, 64, 2, 2, 4>;
template <class T, int I>
constexpr bool kAgrees = T::MF == kFragments[I][0] && T::NF == kFragments[I][1] && T::kThreads == kTileThreads[I];
static_assert(kAgrees<Tile0, 0> && kAgrees<Tile1, 1> && kAgrees<Tile2, 2> && kAgrees<Tile3, 3>, "the scales' layout and the launch");

template <Kind KIND, Out OUT>
int launch_product(const Args& p, int tile, hipStream_t stream) {
    switch (tile) {
        case 0:
            if constexpr (KIND != kMx) return launch_tiles<KIND, OUT, Tile0>(p, stream);
            return NVFP4_ERR_SHAPE;                                  // takes its scales laid out
        case 1: return launch_tiles<KIND, OUT, Tile1>(p, stream);
        case 2: return launch_tiles<KIND, OUT, Tile2>(p, stream);
        default:
            if constexpr (OUT != kGate && OUT != kGatePartial) return launch_tiles<KIND, OUT, Tile3>(p, stream);
            return NVFP4_ERR_SHAPE;                                  // kGate has no plan with it
    }
}

// out = scale * (the parts' sums [parts, count], added in order); values from `first` on go to out2.
int join_parts(const float* part, int parts, int64_t count, const float* scale, void* out, int f32, int64_t first, void* out2,
               hipStream_t stream);

// A product whose sums are stored (kSums, kTwoRows): split where the plan says so, the parts' sums in `partial`.
template <Kind KIND, Out OUT = kSums>
int run_sums(Args p, float* partial, hipStream_t stream) {
    const Plan plan = plan_product<KIND, OUT>(p.m, p.n, p.inner);
    p.parts = plan.parts;
    if (plan.parts == 1) return launch_product<KIND, OUT>(p, plan.tile, stream);
    void* out = p.out;
    p.out = partial;
    if (const int rc = launch_product<KIND, kPartial>(p, plan.tile, stream)) return rc;
    return join_parts(partial, plan.parts, p.m * p.n, p.scale, out, p.out_f32, OUT == kTwoRows ? p.half_rows * p.n : p.m * p.n,
                      p.out2, stream);
}

}  // namespace product_host
