// Host side of the matrix products: the checks that every product shares, the plan of its tiles, and
// the kernels that bring an operand into the form the tiles read.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "nvfp4ss.h"
#include "tile_product.h"

namespace product_host {

using namespace tile_product;

// A tile's loads take 32-bit offsets from its first row: 256 rows of this many bfloat16 values stay
// below the 2 GiB window.
constexpr int64_t kMaxWidth = (int64_t)1 << 20, kMaxLd = (int64_t)1 << 21;
constexpr int64_t kMaxRows = (int64_t)1 << 40;

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
int pack_scale_rows(const uint8_t* src, int64_t rows, int64_t width, uint8_t* dst, int64_t dst_ld, hipStream_t stream);

// Fills in the tiles and steps of p and launches; p's operands, outer indexes and outputs are set.
template <Kind KIND, Layout LA, Layout LB, Pair PAIR, Out OUT, class T>
int launch_product(Args p, hipStream_t stream) {
    constexpr int kStepValues = KIND == kMx ? 256 : 64;
    p.steps = ceil_div(p.inner, kStepValues) * (PAIR == kPairInner ? 2 : 1);
    p.tiles_m = ceil_div(p.m, T::M);
    p.tiles_n = ceil_div(p.n, PAIR == kPairOuter ? T::N / 2 : T::N);
    if (p.parts < 1) p.parts = 1;
    p.split_steps = ceil_div(p.steps, p.parts);
    if (p.tiles_m > 0x7FFFFFFF || p.tiles_m * p.tiles_n > 0x7FFFFFFF / p.parts) return NVFP4_ERR_SHAPE;
    if (p.tiles_m * p.tiles_n == 0) return NVFP4_OK;
    hipLaunchKernelGGL((product_kernel<KIND, LA, LB, PAIR, OUT, T>), dim3((unsigned)(p.tiles_m * p.tiles_n * p.parts)),
                       dim3(T::kThreads), 0, stream, p);
    return launched();
}

}  // namespace product_host
