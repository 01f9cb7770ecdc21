// Microscaled FP4 (OCP MX, MXFP4) on AMD Instinct MI355X (gfx950): E2M1 values in blocks of 32 along
// a row with one E8M0 scale each, the form that gfx950's matrix instructions multiply directly.
//   E = floor(log2 max|x|) - 2 over the block (so that the maximum lies in [4, 8) scales), clamped to
//   -127 .. 127; q_i = RNE_E2M1(x_i 2^-E), saturating at 6.
// Both kernels move bytes: 8 values a lane (16 bytes of bfloat16 in, 4 bytes of nibbles out), the four
// lanes of a block share its maximum through lane permutes, and nothing is kept in LDS.  [8192, 14336] bfloat16: 48 us to
// quantize, 61 to expand (6.2 and 4.9 TB/s).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "launch_limit.h"
#include "nvfp4ss.h"
#include "tile_product.h"

namespace {

using tile_product::pack_bf16;
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 32, kPer = 8, kThreads = 256;

__device__ __forceinline__ float bf16_f32(uint32_t bits) { return __uint_as_float(bits << 16); }

// The largest |x| bits over the four lanes of a block.
__device__ __forceinline__ uint32_t block_top(uint32_t v) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
    v = v > o ? v : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);            // lanes 2 3 0 1
    return v > o ? v : o;
}

// Quantizes the 8 values a lane holds; returns their nibbles and the block's scale code.
__device__ __forceinline__ uint32_t quantize8(const float (&v)[kPer], int& code) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = a > top ? a : top;
    }
    const int e = (int)(block_top(top) >> 23);           // 127 + floor(log2 max|x|); 255: an infinity or a NaN
    code = e == 255 ? 255 : e > 2 ? e - 2 : 0;
    // the conversion divides by 2^(exponent field - 127), also for the field 0, and rounds to nearest even
    const float s = __uint_as_float((uint32_t)code << 23);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], s, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], s, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], s, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], s, 3);
    return q;
}

// WHOLE: cols % 32 == 0, so the tensor is a run of blocks and a lane's values are 8 aligned ones.
// Otherwise rows are taken as filled up to whole blocks, row_units units of 8 each, with zeros past cols.
template <typename In, bool WHOLE>
__global__ __launch_bounds__(kThreads) void mx_quant_kernel(const In* __restrict__ x, int64_t units, int64_t cols,
                                                            int64_t row_units, uint32_t* __restrict__ q,
                                                            uint8_t* __restrict__ scales) {
    int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    float v[kPer];
    if constexpr (WHOLE) {
        if (u >= units) return;                          // whole blocks of lanes: units is a multiple of 4
        if constexpr (sizeof(In) == 2) {
            const uint4 w = *reinterpret_cast<const uint4*>(x + u * kPer);
            const uint32_t p[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_f32(p[i] & 0xFFFFu);
                v[2 * i + 1] = __uint_as_float(p[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 w = *reinterpret_cast<const float4*>(x + u * kPer + h * 4);
                v[4 * h] = w.x, v[4 * h + 1] = w.y, v[4 * h + 2] = w.z, v[4 * h + 3] = w.w;
            }
        }
    } else {
        if (u >= units) return;
        const int64_t row = u / row_units, c = u % row_units * kPer;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const In w = c + i < cols ? x[row * cols + c + i] : In(0);
            if constexpr (sizeof(In) == 2) v[i] = bf16_f32(w);
            else v[i] = w;
        }
    }
    int code;
    const uint32_t n = quantize8(v, code);
    q[u] = n;
    if (u % 4 == 0) scales[u / 4] = (uint8_t)code;
}

template <typename Out, bool WHOLE>
__global__ __launch_bounds__(kThreads) void mx_dequant_kernel(const uint32_t* __restrict__ q,
                                                              const uint8_t* __restrict__ scales, int64_t units,
                                                              int64_t cols, int64_t row_units, Out* __restrict__ out) {
    const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (u >= units) return;
    const uint32_t code = scales[u / 4], n = q[u];
    const float s = __uint_as_float(code << 23);
    f32x2 d[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 1),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 3)};
    if (code == 255) {
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i][0] = d[i][1] = __uint_as_float(0x7FC00000u);
    }
    if constexpr (WHOLE) {
        if constexpr (sizeof(Out) == 2) {
            *reinterpret_cast<uint4*>(out + u * kPer) = make_uint4(pack_bf16(d[0][0], d[0][1]), pack_bf16(d[1][0], d[1][1]),
                                                                   pack_bf16(d[2][0], d[2][1]), pack_bf16(d[3][0], d[3][1]));
        } else {
            *reinterpret_cast<float4*>(out + u * kPer) = make_float4(d[0][0], d[0][1], d[1][0], d[1][1]);
            *reinterpret_cast<float4*>(out + u * kPer + 4) = make_float4(d[2][0], d[2][1], d[3][0], d[3][1]);
        }
    } else {
        const int64_t row = u / row_units, c = u % row_units * kPer;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (c + i >= cols) break;
            const float f = d[i / 2][i % 2];
            if constexpr (sizeof(Out) == 2) out[row * cols + c + i] = (uint16_t)pack_bf16(f, f);
            else out[row * cols + c + i] = f;
        }
    }
}

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct Shape { int64_t units, row_units, groups; };

int shape_of(int64_t rows, int64_t cols, Shape& s) {
    if (rows < 0 || cols < 0 || cols > INT64_MAX / 2 - kBlock) return NVFP4_ERR_SHAPE;
    s.row_units = (cols + kBlock - 1) / kBlock * (kBlock / kPer);
    if (s.row_units && rows > most_groups(kThreads) * kThreads / s.row_units) return NVFP4_ERR_SHAPE;
    s.units = rows * s.row_units;
    s.groups = (s.units + kThreads - 1) / kThreads;
    return NVFP4_OK;
}

}  // namespace

extern "C" {

int mxfp4_quant(const void* x, int dtype, int64_t rows, int64_t cols, uint8_t* q, uint8_t* scales, void* stream) {
    if (dtype != NVFP4_IN_F32 && dtype != NVFP4_IN_BF16) return NVFP4_ERR_DTYPE;
    Shape s;
    if (const int rc = shape_of(rows, cols, s)) return rc;
    if (s.units == 0) return NVFP4_OK;
    if (!x || !q || !scales) return NVFP4_ERR_NULL;
    if (!aligned(x, 16) || !aligned(q, 16)) return NVFP4_ERR_ALIGN;
    auto launch = [&](auto kernel, auto* xt) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)s.groups), dim3(kThreads), 0, (hipStream_t)stream, xt, s.units, cols,
                           s.row_units, reinterpret_cast<uint32_t*>(q), scales);
    };
    const bool whole = cols % kBlock == 0;
    if (dtype == NVFP4_IN_F32)
        launch(whole ? mx_quant_kernel<float, true> : mx_quant_kernel<float, false>, static_cast<const float*>(x));
    else
        launch(whole ? mx_quant_kernel<uint16_t, true> : mx_quant_kernel<uint16_t, false>,
               static_cast<const uint16_t*>(x));
    return hipGetLastError() == hipSuccess ? NVFP4_OK : NVFP4_ERR_HIP;
}

int mxfp4_dequant(const uint8_t* q, const uint8_t* scales, int64_t rows, int64_t cols, int out_dtype, void* out,
                  void* stream) {
    if (out_dtype != NVFP4_IN_F32 && out_dtype != NVFP4_IN_BF16) return NVFP4_ERR_DTYPE;
    Shape s;
    if (const int rc = shape_of(rows, cols, s)) return rc;
    if (s.units == 0) return NVFP4_OK;
    if (!q || !scales || !out) return NVFP4_ERR_NULL;
    if (!aligned(q, 16) || !aligned(out, 16)) return NVFP4_ERR_ALIGN;
    auto launch = [&](auto kernel, auto* o) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)s.groups), dim3(kThreads), 0, (hipStream_t)stream,
                           reinterpret_cast<const uint32_t*>(q), scales, s.units, cols, s.row_units, o);
    };
    const bool whole = cols % kBlock == 0;
    if (out_dtype == NVFP4_IN_F32)
        launch(whole ? mx_dequant_kernel<float, true> : mx_dequant_kernel<float, false>, static_cast<float*>(out));
    else
        launch(whole ? mx_dequant_kernel<uint16_t, true> : mx_dequant_kernel<uint16_t, false>,
               static_cast<uint16_t*>(out));
    return hipGetLastError() == hipSuccess ? NVFP4_OK : NVFP4_ERR_HIP;
}

}  // extern "C"
