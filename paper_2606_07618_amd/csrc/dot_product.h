// Products with one to four activation rows (a decode step): reading the weights is all there is to do, so a wave
// reads whole stretches of a row, its lanes along the contraction, and has many rows in flight.
//
// NVFP4: what else stands in its way are instructions, so each weight pair costs one conversion and one two-way dot
// product a row.  A lane holds 32 values' activations in registers and goes down eight weight rows, whose loads are
// all in flight at once.  The values of a block are summed before the sum is multiplied by the block's
// scale, so scales cost an instruction a block.  They enter 2^-7 as large, and the scale 2^7, both exact: so the sum of a
// block of the largest activations stays within binary32 where the outputs do.
//   y[m][n] = S sum_blocks s sum_j q_j x_j, sums in binary32.
// (A matrix instruction would need the weights times their scales, twice the conversions, and of its 16 columns 12
// to 15 would be empty: one row, [4096, 14336], 14.8 us in place of 9.0, 3.7 TB/s.)
#pragma once

#include "tile_product.h"

namespace dot_product {

using namespace tile_product;
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

using product_plan::kDotRows;
constexpr int kMostRows = kDotRows;
constexpr int kWaves = 8, kSpan = kLanes * 32;   // values of the contraction that a wave's lanes cover
constexpr int kRows = 8;                         // weight rows a wave goes down

struct Args {
    const char* q;
    const uint8_t* scales;
    const char* x;                               // [m, ldx bytes]
    int64_t ldx, n, k;
    int shift, along;                            // along: waves of a workgroup along the contraction, 1, 2, 4 or 8
    const float* scale;
    void* out;
    int out_f32;
};

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
}

constexpr int kUp = 7;                           // of a scale; 32 values of up to 6 make 1.5 2^kUp

// Eight values of a word of nibbles, times 2^-kUp, against eight activations.
__device__ __forceinline__ float dot8(uint32_t n, i32x4 x, float c) {
    constexpr float down = 1.0f / (1 << kUp);
    c = dot2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(n, down, 0)), (uint32_t)x[0], c);
    c = dot2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(n, down, 1)), (uint32_t)x[1], c);
    c = dot2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(n, down, 2)), (uint32_t)x[2], c);
    return dot2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(n, down, 3)), (uint32_t)x[3], c);
}

// Sums over the two halves of a wave (of its rows of 16) of two values at once: the first value's in the lower
// lanes, the second's in the upper ones.
__device__ __forceinline__ float fold32(float a, float b) {
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold16(float a, float b) {
    const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
// The sum over each row of 16 lanes, in all of them.
__device__ __forceinline__ float sum16(float v) {
    v = add_dpp<0xB1>(v);                        // lanes 1 0 3 2
    v = add_dpp<0x4E>(v);                        // lanes 2 3 0 1
    v = add_dpp<0x141>(v);                       // half rows mirrored
    return add_dpp<0x140>(v);                    // rows mirrored
}

// M: activation rows.  EVEN: k is a multiple of 32.  PAIRS: blocks of 16.
template <int M, bool EVEN, bool PAIRS>
__global__ __launch_bounds__(kWaves * kLanes) void dot_kernel(Args p) {
    __shared__ float sums[kWaves][M][kRows];
    const int tid = threadIdx.x, lane = tid % kLanes;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int along = p.along, part = wave % along, group = wave / along;
    const int64_t n0 = (int64_t)blockIdx.x * (kRows * (kWaves / along)) + group * kRows;
    const uint32_t q_ld = (uint32_t)(p.k / 2), s_ld = (uint32_t)(p.k >> p.shift), k = (uint32_t)p.k;
    const __amdgpu_buffer_rsrc_t rq = window(p.q + n0 * q_ld), rs = window(p.scales + n0 * s_ld), rx = window(p.x);
    const int64_t left = p.n - n0;               // rows of this wave that there are: uniform

    float acc[M][kRows];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < kRows; ++r) acc[m][r] = 0.0f;

    for (uint32_t at = (uint32_t)part * kSpan; at < k; at += (uint32_t)along * kSpan) {
        const uint32_t v = at + lane * 32;       // this lane's 32 values
        const bool in0 = v < k, in1 = EVEN ? in0 : v + 16 < k;
        i32x4 x[M][4], w[kRows];
        uint32_t s[kRows];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[m][j] = load16(rx, (j < 2 ? in0 : in1) ? (uint32_t)m * (uint32_t)p.ldx + v * 2 + j * 16 : kOutside);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool row = r < left;
            const uint32_t q_at = r * q_ld + v / 2, s_at = r * s_ld + (v >> p.shift);
            if constexpr (EVEN) {
                w[r] = load16(rq, row && in0 ? q_at : kOutside);
            } else {
                const i32x2 lo = load8(rq, row && in0 ? q_at : kOutside), hi = load8(rq, row && in1 ? q_at + 8 : kOutside);
                w[r] = i32x4{lo[0], lo[1], hi[0], hi[1]};
            }
            if constexpr (!PAIRS) s[r] = load1(rs, row && in0 ? s_at : kOutside);
            else if constexpr (EVEN)
                s[r] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(row && in0 ? s_at : kOutside), 0, 0);
            else s[r] = load1(rs, row && in0 ? s_at : kOutside) | load1(rs, row && in1 ? s_at + 1 : kOutside) << 8;
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float s0 = e4m3_f32<kUp>(s[r]), s1 = PAIRS ? e4m3_f32<kUp>(s[r] >> 8) : s0;
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const float lo = dot8((uint32_t)w[r][1], x[m][1], dot8((uint32_t)w[r][0], x[m][0], 0.0f));
                if constexpr (PAIRS) {
                    const float hi = dot8((uint32_t)w[r][3], x[m][3], dot8((uint32_t)w[r][2], x[m][2], 0.0f));
                    acc[m][r] = fmaf(hi, s1, fmaf(lo, s0, acc[m][r]));
                } else {
                    acc[m][r] = fmaf(dot8((uint32_t)w[r][3], x[m][3], dot8((uint32_t)w[r][2], x[m][2], lo)), s0, acc[m][r]);
                }
            }
        }
    }

    // each row of 16 lanes gets the sums of weight rows 0 to 3 or 4 to 7
#pragma unroll
    for (int m = 0; m < M; ++m) {
        static_assert(kRows == 8, "two folds and a pair");
        const float a = sum16(fold16(fold32(acc[m][0], acc[m][2]), fold32(acc[m][1], acc[m][3])));
        const float b = sum16(fold16(fold32(acc[m][4], acc[m][6]), fold32(acc[m][5], acc[m][7])));
        if (lane % 16 == 0) {
            sums[wave][m][lane / 16] = a;
            sums[wave][m][4 + lane / 16] = b;
        }
    }
    __syncthreads();
    const int outs = M * kRows * (kWaves / along);
    if (tid >= outs) return;
    const int r = tid % kRows, m = tid / kRows % M, of = tid / (kRows * M);
    float v = 0.0f;
    for (int a = 0; a < along; ++a) v += sums[of * along + a][m][r];
    const int64_t n = (int64_t)blockIdx.x * (kRows * (kWaves / along)) + of * kRows + r;
    if (n >= p.n) return;
    v *= *p.scale;
    if (p.out_f32) static_cast<float*>(p.out)[m * p.n + n] = v;
    else static_cast<uint16_t*>(p.out)[m * p.n + n] = (uint16_t)pack_bf16(v, v);
}

// The gated block in the same way, bfloat16 weights: a lane holds eight values of the contraction and goes down
// kGatedRows rows of both matrices.
constexpr int kGatedRows = 8, kGatedSpan = kLanes * 8;

struct GatedArgs {
    const char *wg, *wu;                         // [n, ldw bytes]
    const char* x;                               // [m, ldx bytes]
    int64_t ldw, ldx, n, k;
    int along;
    void *h, *gate, *up;
};

template <int M>
__global__ __launch_bounds__(kWaves * kLanes) void gated_dot_kernel(GatedArgs p) {
    __shared__ float sums[kWaves][2][M][kGatedRows];
    const int tid = threadIdx.x, lane = tid % kLanes;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int along = p.along, part = wave % along, group = wave / along;
    const int64_t rows = kGatedRows * (kWaves / along), n0 = blockIdx.x * rows + group * kGatedRows, left = p.n - n0;
    const __amdgpu_buffer_rsrc_t rw[2] = {window(p.wg + n0 * p.ldw), window(p.wu + n0 * p.ldw)}, rx = window(p.x);
    const uint32_t k = (uint32_t)p.k;

    float acc[2][M][kGatedRows];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < kGatedRows; ++r) acc[b][m][r] = 0.0f;

    for (uint32_t at = (uint32_t)part * kGatedSpan; at < k; at += (uint32_t)along * kGatedSpan) {
        const uint32_t v = at + lane * 8;        // rows hold whole groups of eight, zeros past k
        i32x4 x[M], w[2][kGatedRows];
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = load16(rx, v < k ? (uint32_t)m * (uint32_t)p.ldx + v * 2 : kOutside);
#pragma unroll
        for (int r = 0; r < kGatedRows; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                w[b][r] = load16(rw[b], r < left && v < k ? (uint32_t)r * (uint32_t)p.ldw + v * 2 : kOutside);
#pragma unroll
        for (int r = 0; r < kGatedRows; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[b][m][r] = dot2((uint32_t)w[b][r][j], (uint32_t)x[m][j], acc[b][m][r]);
    }

#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int m = 0; m < M; ++m) {
            static_assert(kGatedRows == 8, "two folds and a pair");
            const float* a = acc[b][m];
            const float lo = sum16(fold16(fold32(a[0], a[2]), fold32(a[1], a[3])));
            const float hi = sum16(fold16(fold32(a[4], a[6]), fold32(a[5], a[7])));
            if (lane % 16 == 0) {
                sums[wave][b][m][lane / 16] = lo;
                sums[wave][b][m][4 + lane / 16] = hi;
            }
        }
    __syncthreads();
    if (tid >= M * kGatedRows * (kWaves / along)) return;
    const int r = tid % kGatedRows, m = tid / kGatedRows % M, of = tid / (kGatedRows * M);
    const int64_t n = blockIdx.x * rows + of * kGatedRows + r;
    if (n >= p.n) return;
    float g = 0.0f, u = 0.0f;
    for (int a = 0; a < along; ++a) {
        g += sums[of * along + a][0][m][r];
        u += sums[of * along + a][1][m][r];
    }
    const float h = silu(g) * u;
    static_cast<uint16_t*>(p.h)[m * p.n + n] = (uint16_t)pack_bf16(h, h);
    if (p.gate) {
        static_cast<uint16_t*>(p.gate)[m * p.n + n] = (uint16_t)pack_bf16(g, g);
        static_cast<uint16_t*>(p.up)[m * p.n + n] = (uint16_t)pack_bf16(u, u);
    }
}

// Waves of a workgroup along the contraction, for spans of `span` values.
inline int waves_along(int64_t k, int span) {
    int along = 1;
    while (along < kWaves && (int64_t)along * span < k) along *= 2;
    return along;
}

template <int M>
void launch_gated_dot(const GatedArgs& p, hipStream_t stream) {
    const int64_t rows = kGatedRows * (kWaves / p.along);
    hipLaunchKernelGGL((gated_dot_kernel<M>), dim3((unsigned)((p.n + rows - 1) / rows)), dim3(kWaves * kLanes), 0, stream, p);
}

template <int M>
void launch_dot(const Args& p, hipStream_t stream) {
    const bool even = p.k % 32 == 0, pairs = p.shift == 4;
    auto kernel = even ? (pairs ? dot_kernel<M, true, true> : dot_kernel<M, true, false>) : dot_kernel<M, false, true>;
    const int64_t rows = kRows * (kWaves / p.along);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n + rows - 1) / rows)), dim3(kWaves * kLanes), 0, stream, p);
}

}  // namespace dot_product
