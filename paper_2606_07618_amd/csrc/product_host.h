// Host side of the matrix products: the checks that every product shares, the launch of its planned tiles, and
// the kernels that bring an operand into the form the tiles read.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "nvfp4ss.h"
#include "product_plan.h"
#include "tile_product.h"

namespace product_host {

using namespace product_plan;
using namespace tile_product;

// A tile's loads take 32-bit offsets from its first row: 256 rows of this many bfloat16 values stay
// below the 2 GiB window.
constexpr int64_t kMaxWidth = (int64_t)1 << 20, kMaxLd = (int64_t)1 << 21;
constexpr int64_t kMaxRows = (int64_t)1 << 36;      // workspace sizes stay within 63 bits

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

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

// Fills in the tiles and steps of p and launches; p's operands, outer indexes and outputs are set.
template <Kind KIND, Out OUT, class T>
int launch_tiles(Args p, hipStream_t stream) {
    p.steps = ceil_div(p.inner, kStepValues<KIND>);
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
