// Microscaled products with few rows of activations and weights too small to keep the chip busy with tiles: nothing is
// staged and nothing waits for a neighbour.  A workgroup owns 16 weight rows; its waves
// take turns along the contraction, each loading weights straight into the registers of its matrix instructions (16
// rows by four lanes of 16 bytes), the activations' side of the instruction from the caches, kUnroll such pieces in
// flight; one exchange through LDS adds the waves' sums, in a fixed order.  One row, [4096, 4096]: 5.2 us (1.7 TB/s,
// most of it the way to memory and back), 11.2 with tiles; [4096, 14336] 10.9 (2.9 TB/s) and 15; with tiles enough,
// [28672, 8192], 36 and 31.
// Lanes past the operands' ends load nothing (kOutside) and multiply zeros.
#pragma once

#include "tile_product.h"

namespace thin_product {

using namespace tile_product;
using product_plan::kThinRows;
constexpr int kRows = kThinRows;                 // of the activations, at most

struct Args {
    const char *w, *x;                           // [n, k], [m, k] nibbles
    const uint8_t *w_scales, *x_scales;
    int64_t n, k;                                // k: values, whole blocks
    int m;
    void* out;
    int out_f32;
};

constexpr int kWaves = 8, kUnroll = 4;
constexpr uint32_t kPiece = 128;                 // values of a row in one load of a wave

__global__ __launch_bounds__(kWaves * kLanes) void thin_kernel(Args p) {
    __shared__ f32x4 sums[kWaves][kLanes];
    const int tid = threadIdx.x, lane = tid % kLanes, g = lane / 16, i = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int64_t n0 = (int64_t)blockIdx.x * 16, ld = p.k / 2, scale_ld = p.k / 32;
    const __amdgpu_buffer_rsrc_t rw = window(p.w + n0 * ld), rx = window(p.x),
                                 rs = window(p.w_scales + n0 * scale_ld), rxs = window(p.x_scales);
    const bool row_in = n0 + i < p.n, m_in = i < p.m;
    const uint32_t k = (uint32_t)p.k, row = (uint32_t)i * (uint32_t)ld, scale_row = (uint32_t)i * (uint32_t)scale_ld;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t at = (uint32_t)wave * kUnroll * kPiece; at < k; at += kWaves * kUnroll * kPiece) {
        i32x4 a[kUnroll], x[kUnroll];
        uint32_t s[kUnroll], t[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint32_t v = at + u * kPiece + g * 32;
            const bool wi = row_in && v < k, xi = m_in && v < k;
            a[u] = load16(rw, wi ? row + v / 2 : kOutside);
            x[u] = load16(rx, xi ? row + v / 2 : kOutside);
            s[u] = load1(rs, wi ? scale_row + v / 32 : kOutside);
            t[u] = load1(rxs, xi ? scale_row + v / 32 : kOutside);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const i32x8 wa = {a[u][0], a[u][1], a[u][2], a[u][3], 0, 0, 0, 0}, wx = {x[u][0], x[u][1], x[u][2], x[u][3], 0, 0, 0, 0};
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wx, acc, 4, 4, 0, (int)s[u], 0, (int)t[u]);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    acc = sums[0][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) acc += sums[w][lane];
    // a lane holds outputs n0 + 4 g .. + 3 of activation row i
    const int64_t n = n0 + g * 4;
    if (m_in) store4(p.out, p.out_f32, (int64_t)i * p.n + n, p.n - n, p.n % 4 == 0, acc);
}

inline void launch_thin(const Args& p, hipStream_t stream) {
    hipLaunchKernelGGL(thin_kernel, dim3((unsigned)((p.n + 15) / 16)), dim3(kWaves * kLanes), 0, stream, p);
}

}  // namespace thin_product
