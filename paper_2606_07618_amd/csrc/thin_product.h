// Products with few rows of activations (one token, a decode step of a small batch): reading the weights is
// all there is, so nothing is staged and nothing waits for a neighbour.  A workgroup owns 16 weight rows;
// its waves take turns along the contraction, each loading weights straight into the registers of its matrix
// instructions (16 rows by four lanes of 16 bytes), the activations' side of the instruction from the caches,
// kUnroll such pieces in flight; one exchange through LDS adds the waves' sums, in a fixed order.
// Lanes past the operands' ends load nothing (kOutside) and multiply zeros.
#pragma once

#include "tile_product.h"

namespace thin_product {

using namespace tile_product;
constexpr int kRows = 16;                        // of the activations, at most

// What multiplies: bfloat16 weights (two matrices, gated), or both sides microscaled.
enum Weights { kGated, kMicroscaled };

struct Args {
    const char *w, *w2;                          // [n, ldw bytes]
    const uint8_t* w_scales;                     // [n, w_scale_ld]
    int64_t ldw, w_scale_ld;
    const char* x;                               // [m, ldx bytes]
    const uint8_t* x_scales;
    int64_t ldx;
    int64_t n, k;                                // k: values
    int m;
    void *out, *out2, *out3;
    int out_f32;
};

template <Weights W, int WAVES, int kUnroll>
__global__ __launch_bounds__(WAVES * kLanes) void thin_kernel(Args p) {
    constexpr int kAcc = W == kGated ? 2 : 1;
    __shared__ f32x4 sums[WAVES][kAcc][kLanes];
    const int tid = threadIdx.x, lane = tid % kLanes, g = lane / 16, i = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const __amdgpu_buffer_rsrc_t rw = window(p.w + n0 * p.ldw), rx = window(p.x);
    const bool row_in = n0 + i < p.n, m_in = i < p.m;
    const uint32_t w_row = (uint32_t)i * (uint32_t)p.ldw, x_row = (uint32_t)i * (uint32_t)p.ldx;
    const uint32_t k = (uint32_t)p.k;
    f32x4 acc[kAcc];
#pragma unroll
    for (int a = 0; a < kAcc; ++a) acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    if constexpr (W == kGated) {
        const __amdgpu_buffer_rsrc_t rw2 = window(p.w2 + n0 * p.ldw);
        constexpr uint32_t kPiece = 32;                        // values of a row in one load
        for (uint32_t at = (uint32_t)wave * kUnroll * kPiece; at < k; at += WAVES * kUnroll * kPiece) {
            i32x4 a[kUnroll], b[kUnroll], x[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const uint32_t v = at + u * kPiece + g * 8;
                a[u] = load16(rw, row_in && v < k ? w_row + v * 2 : kOutside);
                b[u] = load16(rw2, row_in && v < k ? w_row + v * 2 : kOutside);
                x[u] = load16(rx, m_in && v < k ? x_row + v * 2 : kOutside);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const bf16x8 xv = __builtin_bit_cast(bf16x8, x[u]);
                acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u]), xv, acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[u]), xv, acc[1], 0, 0, 0);
            }
        }
    } else {
        const __amdgpu_buffer_rsrc_t rs = window(p.w_scales + n0 * p.w_scale_ld), rxs = window(p.x_scales);
        const uint32_t s_row = (uint32_t)i * (uint32_t)p.w_scale_ld;   // the activations' scales have rows as long
        constexpr uint32_t kPiece = 128;
        for (uint32_t at = (uint32_t)wave * kUnroll * kPiece; at < k; at += WAVES * kUnroll * kPiece) {
            i32x4 a[kUnroll], x[kUnroll];
            uint32_t s[kUnroll], t[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const uint32_t v = at + u * kPiece + g * 32;
                const bool wi = row_in && v < k, xi = m_in && v < k;
                a[u] = load16(rw, wi ? w_row + v / 2 : kOutside);
                x[u] = load16(rx, xi ? x_row + v / 2 : kOutside);
                s[u] = load1(rs, wi ? s_row + v / 32 : kOutside);
                t[u] = load1(rxs, xi ? s_row + v / 32 : kOutside);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const i32x8 wa = {a[u][0], a[u][1], a[u][2], a[u][3], 0, 0, 0, 0}, wx = {x[u][0], x[u][1], x[u][2], x[u][3], 0, 0, 0, 0};
                acc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wx, acc[0], 4, 4, 0, (int)s[u], 0, (int)t[u]);
            }
        }
    }

#pragma unroll
    for (int a = 0; a < kAcc; ++a) sums[wave][a][lane] = acc[a];
    __syncthreads();
    if (wave > 0) return;
    f32x4 v[kAcc];
#pragma unroll
    for (int a = 0; a < kAcc; ++a) {
        v[a] = sums[0][a][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v[a] += sums[w][a][lane];
    }
    // a lane holds outputs n0 + 4 g .. + 3 of activation row i
    if (!m_in) return;
    const int64_t n = n0 + g * 4, left = p.n - n, to = (int64_t)i * p.n + n;
    const bool vec = p.n % 4 == 0;
    if constexpr (W == kGated) {
        f32x4 h;
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = silu(v[0][r]) * v[1][r];
        store4(p.out, 0, to, left, vec, h);
        if (p.out2) {
            store4(p.out2, 0, to, left, vec, v[0]);
            store4(p.out3, 0, to, left, vec, v[1]);
        }
    } else {
        store4(p.out, p.out_f32, to, left, vec, v[0]);
    }
}

template <Weights W, int WAVES, int kUnroll>
void launch_thin(const Args& p, hipStream_t stream) {
    hipLaunchKernelGGL((thin_kernel<W, WAVES, kUnroll>), dim3((unsigned)((p.n + 15) / 16)), dim3(WAVES * kLanes), 0, stream, p);
}

}  // namespace thin_product
