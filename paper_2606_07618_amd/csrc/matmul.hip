// Matrix products with 4-bit weights on AMD Instinct MI355X (gfx950).
//   NVFP4 weights W = q s S [n, k], activations in bfloat16:  y = x W^T,  dx = dy W
//   microscaled FP4 (E8M0 scale for each 32 values):          y = A B^T,  dx = dy B
#include "product_host.h"
#include "dot_product.h"
#include "stream_product.h"
#include "thin_product.h"

namespace product_host {

namespace {

constexpr int kPackThreads = 256;

__global__ __launch_bounds__(kPackThreads) void pack_kernel(const uint16_t* __restrict__ src, int64_t count, int64_t width,
                                                            int64_t ld, uint16_t* __restrict__ dst, int64_t dst_ld) {
    for (int64_t i = (int64_t)blockIdx.x * kPackThreads + threadIdx.x; i < count; i += (int64_t)gridDim.x * kPackThreads) {
        const int64_t r = i / dst_ld, c = i % dst_ld;
        dst[i] = c < width ? src[r * ld + c] : (uint16_t)0;
    }
}

// Sums of parts of the contraction.
template <bool VEC>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const float* __restrict__ part, int parts, int64_t count,
                                                            const float* __restrict__ scale, void* __restrict__ out,
                                                            int f32, int64_t first, void* __restrict__ out2) {
    constexpr int kPer = VEC ? 4 : 1;
    const int64_t at = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) * kPer;
    if (at >= count) return;
    float v[kPer] = {};
    for (int p = 0; p < parts; ++p) {
        const float* from = part + p * count + at;
        if constexpr (VEC) {
            const float4 w = *reinterpret_cast<const float4*>(from);
            v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
        } else {
            v[0] += *from;
        }
    }
    const float s = scale ? *scale : 1.0f;
    void* to = at < first ? out : out2;
    const int64_t place = at < first ? at : at - first;
    if constexpr (VEC) store4(to, f32, place, 4, true, f32x4{v[0], v[1], v[2], v[3]} * s);
    else store4(to, f32, place, 1, false, f32x4{v[0] * s, 0.0f, 0.0f, 0.0f});
}

}  // namespace

int pack_bf16_rows(const void* src, int64_t rows, int64_t width, int64_t ld, void* dst, hipStream_t stream) {
    const int64_t count = rows * packed_ld(width), groups = ceil_div(count, kPackThreads);
    if (count == 0) return NVFP4_OK;
    hipLaunchKernelGGL(pack_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(kPackThreads), 0, stream,
                       static_cast<const uint16_t*>(src), count, width, ld, static_cast<uint16_t*>(dst), packed_ld(width));
    return launched();
}

int join_parts(const float* part, int parts, int64_t count, const float* scale, void* out, int f32, int64_t first, void* out2,
               hipStream_t stream) {
    const bool vec = count % 4 == 0 && first % 4 == 0;
    const int64_t groups = ceil_div(vec ? count / 4 : count, kJoinThreads);
    if (!launchable(groups, kJoinThreads)) return NVFP4_ERR_SHAPE;
    hipLaunchKernelGGL((vec ? join_kernel<true> : join_kernel<false>), dim3((unsigned)groups), dim3(kJoinThreads), 0, stream,
                       part, parts, count, scale, out, f32, first, out2);
    return launched();
}

}  // namespace product_host

namespace {

using namespace product_host;

// ---- weights expanded to bfloat16 -----------------------------------------------------------

// q s of NVFP4 (without S) or q 2^E of microscaled FP4, 8 values a lane, both exact: an E2M1 value has
// two significand bits and an E4M3 scale four, bfloat16 eight; the smallest microscaled value, 2^-128, is a
// multiple of bfloat16's least, 2^-133, and the matrix instructions take such numbers as they are.
template <Kind KIND>
__device__ __forceinline__ uint4 expand8(uint32_t n, uint32_t code) {
    const float s = KIND == kMx ? __uint_as_float(code << 23) : 1.0f, t = KIND == kMx ? 1.0f : e4m3_f32(code);
    f32x2 d[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 1),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, s, 3)};
    if (KIND == kMx && code == 255) d[0] = d[1] = d[2] = d[3] = f32x2{__uint_as_float(0x7FC00000u), __uint_as_float(0x7FC00000u)};
    return make_uint4(pack_bf16(d[0][0] * t, d[0][1] * t), pack_bf16(d[1][0] * t, d[1][1] * t),
                      pack_bf16(d[2][0] * t, d[2][1] * t), pack_bf16(d[3][0] * t, d[3][1] * t));
}

constexpr int kExpandThreads = 256;

// Rows of row_units units of 8 values, a scale for each 2^shift of them; a workgroup expands a piece of one row.
__global__ __launch_bounds__(kExpandThreads) void expand_kernel(const uint32_t* __restrict__ q,
                                                                const uint8_t* __restrict__ scales, uint32_t row_units,
                                                                uint32_t row_groups, int shift, uint4* __restrict__ out) {
    const uint32_t row = blockIdx.x / row_groups, u = blockIdx.x % row_groups * kExpandThreads + threadIdx.x;
    if (u >= row_units) return;
    const int64_t at = (int64_t)row * row_units + u;
    out[at] = expand8<kBf16>(q[at], scales[at >> shift]);
}

int64_t expand_groups(int64_t n, int64_t k) { return n * ceil_div(k / 8, kExpandThreads); }

int expand(const uint8_t* q, const uint8_t* scales, int64_t n, int64_t k, int block, void* out, hipStream_t stream) {
    const int64_t row_units = k / 8, row_groups = ceil_div(row_units, kExpandThreads);
    if (n * row_units == 0) return NVFP4_OK;
    int shift = 1;
    while (8 << shift < block) ++shift;
    hipLaunchKernelGGL(expand_kernel, dim3((unsigned)(n * row_groups)), dim3(kExpandThreads), 0, stream,
                       reinterpret_cast<const uint32_t*>(q), scales, (uint32_t)row_units, (uint32_t)row_groups, shift,
                       static_cast<uint4*>(out));
    return launched();
}

// The same transposed, [k, ld] with zeros from n to ld: as rows of the gradient's contraction.  A workgroup turns 64
// by 128 values in LDS, whose rows are two words longer than their values so that a wave's writes, 16 weight rows
// by four rows of the tile 16 apart, meet in no bank.
constexpr int kTurnN = 64, kTurnK = 128;

template <Kind KIND>
__global__ __launch_bounds__(kExpandThreads) void expand_turned_kernel(const uint8_t* __restrict__ q,
                                                                       const uint8_t* __restrict__ scales, int64_t n,
                                                                       uint32_t k, uint32_t tiles_k, int shift, int64_t ld,
                                                                       uint16_t* __restrict__ out) {
    __shared__ uint32_t tile[kTurnK][kTurnN / 2 + 1];
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_k) * kTurnN;
    const uint32_t k0 = blockIdx.x % tiles_k * kTurnK;
    const int row = threadIdx.x / 4, part = threadIdx.x % 4;             // 16 values of a weight row, 64 apart
    const uint64_t row_at = (uint64_t)(n0 + row) * k;
    constexpr int kPieces = kTurnK / 64;
    uint2 w[kPieces];
    uint32_t code[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const uint32_t at = k0 + p * 64 + part * 16;                     // k is a multiple of 16
        const bool in = n0 + row < n && at < k;
        w[p] = in ? *reinterpret_cast<const uint2*>(q + (row_at + at) / 2) : make_uint2(0u, 0u);
        code[p] = in ? scales[(row_at + at) >> shift] : 0u;
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const uint4 a = expand8<KIND>(w[p].x, code[p]), b = expand8<KIND>(w[p].y, code[p]);
        const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            reinterpret_cast<uint16_t*>(tile[p * 64 + part * 16 + j])[row] = (uint16_t)(v[j / 2] >> (j % 2 * 16));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurnK * kTurnN / 8 / kExpandThreads; ++i) {
        const int c = i * kExpandThreads + threadIdx.x, r = c / (kTurnN / 8), chunk = c % (kTurnN / 8);
        if (k0 + r < k && n0 + chunk * 8 < ld)
            *reinterpret_cast<uint4*>(out + (int64_t)(k0 + r) * ld + n0 + chunk * 8) =
                make_uint4(tile[r][chunk * 4], tile[r][chunk * 4 + 1], tile[r][chunk * 4 + 2], tile[r][chunk * 4 + 3]);
    }
}

int64_t turned_groups(int64_t n, int64_t k) { return ceil_div(n, kTurnN) * ceil_div(k, kTurnK); }

template <Kind KIND>
int expand_turned(const uint8_t* q, const uint8_t* scales, int64_t n, int64_t k, int block, int64_t ld, void* out,
                  hipStream_t stream) {
    const int64_t tiles_k = ceil_div(k, kTurnK), tiles = turned_groups(n, k);
    if (tiles == 0) return NVFP4_OK;
    int shift = 4;
    while (1 << shift < block) ++shift;
    hipLaunchKernelGGL((expand_turned_kernel<KIND>), dim3((unsigned)tiles), dim3(kExpandThreads), 0, stream, q, scales, n,
                       (uint32_t)k, (uint32_t)tiles_k, shift, ld, static_cast<uint16_t*>(out));
    return launched();
}

bool valid_out(int dtype) { return dtype == NVFP4_IN_F32 || dtype == NVFP4_IN_BF16; }

// ---- y = x W^T ------------------------------------------------------------------------------

int64_t linear_workspace(int64_t m, int64_t n, int64_t k) {
    if (m <= kDotRows) return 0;       // one launch, no workspace
    if (m <= kStreamRows) {
        const int parts = stream_parts(m, n, k);
        return parts > 1 ? up(parts * m * n * 4, 256) : 0;
    }
    return up(n * k * 2, 256) + parts_bytes<kBf16>(m, n, k);
}

bool linear_launchable(int64_t m, int64_t n, int64_t k) {
    return m <= kStreamRows || (launchable(expand_groups(n, k), kExpandThreads) && product_launchable<kBf16>(m, n, k));
}

template <int MF>
void launch_stream(const stream_product::Args& p, hipStream_t stream) {
    const dim3 grid((unsigned)(p.tiles_n * p.tiles_m * p.parts)), threads(256 * kWavesK);
    using namespace stream_product;
    const bool wide = p.k % stream_product::kGroup == 0;   // whole groups, whose scales start on whole words
    auto kernel = p.shift == 4 ? (wide ? stream_kernel<MF, kWide16> : p.k % 32 == 0 ? stream_kernel<MF, kPair> : stream_kernel<MF, kOdd>)
                               : p.shift == 5 && wide ? stream_kernel<MF, kWide32> : stream_kernel<MF, kOne>;
    hipLaunchKernelGGL(kernel, grid, threads, 0, stream, p);
}

int run_linear(const void* x, int64_t ldx, const uint8_t* q, const uint8_t* scales, int block, const float* S,
               int64_t m, int64_t n, int64_t k, int out_dtype, void* out, void* ws, hipStream_t stream) {
    const int shift = block == 16 ? 4 : block == 32 ? 5 : block == 64 ? 6 : 7;
    const int f32 = out_dtype == NVFP4_IN_F32;
    if (m <= kDotRows) {
        dot_product::Args t = {};
        t.q = reinterpret_cast<const char*>(q), t.scales = scales, t.x = static_cast<const char*>(x), t.ldx = ldx * 2;
        t.n = n, t.k = k, t.shift = shift, t.scale = S, t.out = out, t.out_f32 = f32;
        t.along = dot_product::waves_along(k, dot_product::kSpan);
        switch (m) {
            case 1: dot_product::launch_dot<1>(t, stream); break;
            case 2: dot_product::launch_dot<2>(t, stream); break;
            case 3: dot_product::launch_dot<3>(t, stream); break;
            default: dot_product::launch_dot<4>(t, stream);
        }
        return launched();
    }
    if (m <= kStreamRows) {
        stream_product::Args t = {};
        t.q = reinterpret_cast<const char*>(q), t.scales = scales, t.x = static_cast<const char*>(x), t.ldx = ldx * 2;
        t.m = m, t.n = n, t.k = k, t.shift = shift, t.scale = S, t.out = out, t.out_f32 = f32;
        t.tiles_n = ceil_div(n, stream_product::kRowsN), t.tiles_m = stream_tiles_m(m);
        t.parts = stream_parts(m, n, k), t.part_values = stream_part_values(k, t.parts);
        float* partial = t.parts > 1 ? static_cast<float*>(ws) : nullptr;
        if (partial) t.out = partial;
        switch (stream_rows_of(m)) {
            case 1: launch_stream<1>(t, stream); break;
            case 2: launch_stream<2>(t, stream); break;
            default: launch_stream<4>(t, stream);
        }
        if (const int rc = launched()) return rc;
        return partial ? join_parts(partial, t.parts, m * n, nullptr, out, f32, m * n, nullptr, stream) : NVFP4_OK;
    }
    Carver c{static_cast<char*>(ws)};
    void* w = c.take(n * k * 2);
    if (const int rc = expand(q, scales, n, k, block, w, stream)) return rc;
    Args p = {};
    p.a.p = static_cast<const char*>(x), p.a.ld = ldx * 2;
    p.b.p = static_cast<const char*>(w), p.b.ld = k * 2;
    p.m = m, p.n = n, p.inner = k, p.scale = S, p.out = out, p.out_ld = n, p.out_f32 = out_dtype == NVFP4_IN_F32;
    return run_sums<kBf16>(p, static_cast<float*>(c.take(0)), stream);
}

// ---- dx = dy W ------------------------------------------------------------------------------
// The weights are expanded with their rows turned, so that both operands hold the contraction along their rows
// ([4096, 14336] x [14336, 4096]: 438 us with the weights as they lie, 360 so).

int64_t grad_workspace(int64_t m, int64_t n, int64_t k, int64_t k32, int64_t ld) {
    Carver c{nullptr};
    c.take(k32 * packed_ld(n) * 2);
    if (needs_pack(n, ld)) c.take(m * packed_ld(n) * 2);
    return c.at + parts_bytes<kBf16>(m, k, n);
}

bool grad_launchable(int64_t m, int64_t n, int64_t k, int64_t k32) {
    return launchable(turned_groups(n, k32), kExpandThreads) && product_launchable<kBf16>(m, k, n);
}

// k32: the width of the weights' rows (k filled up to whole blocks); dx has k columns.
template <Kind KIND>
int run_grad(const void* dy, int64_t ld, const uint8_t* q, const uint8_t* scales, int block, const float* S, int64_t m,
             int64_t n, int64_t k, int64_t k32, int out_dtype, void* out, void* ws, hipStream_t stream) {
    Carver c{static_cast<char*>(ws)};
    void* w = c.take(k32 * packed_ld(n) * 2);
    if (const int rc = expand_turned<KIND>(q, scales, n, k32, block, packed_ld(n), w, stream)) return rc;
    if (needs_pack(n, ld)) {
        void* packed = c.take(m * packed_ld(n) * 2);
        if (const int rc = pack_bf16_rows(dy, m, n, ld, packed, stream)) return rc;
        dy = packed, ld = packed_ld(n);
    }
    Args p = {};
    p.a.p = static_cast<const char*>(dy), p.a.ld = ld * 2;
    p.b.p = static_cast<const char*>(w), p.b.ld = packed_ld(n) * 2;
    p.m = m, p.n = k, p.inner = n, p.scale = S, p.out = out, p.out_ld = k, p.out_f32 = out_dtype == NVFP4_IN_F32;
    return run_sums<kBf16>(p, static_cast<float*>(c.take(0)), stream);
}

// ---- y = A B^T, both microscaled --------------------------------------------------------------

constexpr int kScaleThreads = 256;

struct Scales { const uint8_t* from; uint8_t* to; int64_t rows, groups; int fragments; };

// Both operands' scales as scale_at() lays them out, zeros outside.  A thread takes a step's eight codes of the F rows
// r, 16 + r, .. of a group, and writes them to four lanes.  WORDS: rows are whole words.
template <bool WORDS>
__global__ __launch_bounds__(kScaleThreads) void lay_scales_kernel(Scales a, Scales b, int64_t blocks, int64_t steps) {
    const uint32_t pieces = ((uint32_t)steps * 16 + kScaleThreads - 1) / kScaleThreads;   // of a group's steps
    const uint32_t at = blockIdx.x % pieces * kScaleThreads + threadIdx.x, of = blockIdx.x / pieces;
    const Scales p = of < a.groups ? a : b;
    const int64_t group = of < a.groups ? of : of - a.groups;
    const int r = (int)(at % 16);
    const int64_t step = at / 16;
    if (step >= steps) return;
    const int64_t row0 = group * p.fragments * 16;
    const __amdgpu_buffer_rsrc_t from = window(p.from + row0 * blocks);
    uint32_t code[8][2];                         // of blocks 0 .. 3 and 4 .. 7 of the step
#pragma unroll
    for (int f = 0; f < 8; ++f) {
        const int64_t left = f < p.fragments && row0 + f * 16 + r < p.rows ? blocks - step * 8 : 0;
        const uint32_t offset = (uint32_t)(f * 16 + r) * (uint32_t)blocks + (uint32_t)step * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (WORDS) {
                code[f][h] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(from, (int)(h * 4 < left ? offset + h * 4 : kOutside), 0, 0);
            } else {
                code[f][h] = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) code[f][h] |= load1(from, h * 4 + i < left ? offset + h * 4 + i : kOutside) << i * 8;
            }
        }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t* to = reinterpret_cast<uint32_t*>(p.to + scale_at(group, steps, step, g * 16 + r, p.fragments));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pick = 0x0C0C0400u + g * 0x0101u;
            if (i < p.fragments / 2)
                to[i] = __builtin_amdgcn_perm(code[2 * i][1], code[2 * i][0], pick) |
                        __builtin_amdgcn_perm(code[2 * i + 1][1], code[2 * i + 1][0], pick) << 16;
        }
    }
}

int64_t lay_groups(int64_t m, int64_t n, int64_t blocks, const int* fragments) {
    return (ceil_div(m, 16 * fragments[0]) + ceil_div(n, 16 * fragments[1])) * ceil_div(ceil_div(blocks, 8) * 16, kScaleThreads);
}

int64_t scale_bytes(int64_t rows, int64_t blocks) { return up(rows, 128) * ceil_div(blocks, 8) * 8; }

bool mx_launchable(int64_t m, int64_t n, int64_t blocks) {
    const int* fragments = kFragments[plan_product<kMx, kSums>(m, n, blocks * 32).tile];
    return thin(m, n, blocks) || (product_launchable<kMx>(m, n, blocks * 32) &&
                                  (!lays_scales(m, n, blocks) || launchable(lay_groups(m, n, blocks, fragments), kScaleThreads)));
}

int64_t mx_workspace(int64_t m, int64_t n, int64_t blocks) {
    if (thin(m, n, blocks)) return 0;
    Carver c{nullptr};
    if (lays_scales(m, n, blocks)) {
        c.take(scale_bytes(m, blocks));
        c.take(scale_bytes(n, blocks));
    }
    return c.at + parts_bytes<kMx>(m, n, blocks * 32);
}

int run_mx(const uint8_t* aq, const uint8_t* as, const uint8_t* bq, const uint8_t* bs, int64_t m, int64_t n,
           int64_t blocks, int out_dtype, void* out, void* ws, hipStream_t stream) {
    if (thin(m, n, blocks)) {
        thin_product::Args t = {};
        t.w = reinterpret_cast<const char*>(bq), t.w_scales = bs, t.x = reinterpret_cast<const char*>(aq), t.x_scales = as;
        t.m = (int)m, t.n = n, t.k = blocks * 32, t.out = out, t.out_f32 = out_dtype == NVFP4_IN_F32;
        thin_product::launch_thin(t, stream);
        return launched();
    }
    Carver c{static_cast<char*>(ws)};
    Args p = {};
    p.a.p = reinterpret_cast<const char*>(aq), p.a.ld = blocks * 16, p.a.scales = as, p.a.scale_ld = blocks;
    p.b.p = reinterpret_cast<const char*>(bq), p.b.ld = blocks * 16, p.b.scales = bs, p.b.scale_ld = blocks;
    p.m = m, p.n = n, p.inner = blocks * 32, p.out = out, p.out_ld = n, p.out_f32 = out_dtype == NVFP4_IN_F32;
    if (!lays_scales(m, n, blocks)) return run_sums<kMx>(p, static_cast<float*>(c.take(0)), stream);
    const int* fragments = kFragments[plan_product<kMx, kSums>(m, n, blocks * 32).tile];
    const int64_t steps = ceil_div(blocks, 8);
    const auto scales = [&](const uint8_t* from, int64_t rows, int f) {
        return Scales{from, static_cast<uint8_t*>(c.take(scale_bytes(rows, blocks))), rows, ceil_div(rows, 16 * f), f};
    };
    const Scales a = scales(as, m, fragments[0]), b = scales(bs, n, fragments[1]);
    const int64_t groups = lay_groups(m, n, blocks, fragments);
    if (groups > 0) {
        hipLaunchKernelGGL((blocks % 4 == 0 ? lay_scales_kernel<true> : lay_scales_kernel<false>), dim3((unsigned)groups), dim3(kScaleThreads), 0, stream, a, b, blocks, steps);
        if (const int rc = launched()) return rc;
    }
    p.a.scales = a.to, p.b.scales = b.to;
    return run_sums<kMxLaid>(p, static_cast<float*>(c.take(0)), stream);
}

int check_ws(const void* ws, size_t bytes, int64_t need) {
    if (need > 0 && (!ws || (int64_t)bytes < need)) return NVFP4_ERR_WORKSPACE;
    return aligned(ws, 256) || need == 0 ? NVFP4_OK : NVFP4_ERR_ALIGN;
}

int check_nvfp4(int64_t m, int64_t n, int64_t k, int block) {
    if (block != 16 && block != 32 && block != 64 && block != 128) return NVFP4_ERR_BLOCK;
    if (const int rc = check_dims(m, n, k)) return rc;
    return k % block ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

}  // namespace

extern "C" {

int64_t nvfp4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (const int rc = check_dims(m, n, k)) return rc;
    return linear_workspace(m, n, k);
}

int nvfp4_matmul(const void* x, int64_t ldx, const uint8_t* q, const uint8_t* scales, int block,
                 const float* tensor_scale, int64_t m, int64_t n, int64_t k, int out_dtype, void* out, void* workspace,
                 size_t workspace_bytes, void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_nvfp4(m, n, k, block)) return rc;
    if (ldx < k || ldx > kMaxLd || !linear_launchable(m, n, k)) return NVFP4_ERR_SHAPE;
    if (m == 0 || n == 0) return NVFP4_OK;
    if (!out || !tensor_scale || (k > 0 && (!x || !q || !scales))) return NVFP4_ERR_NULL;
    if (!aligned(x, 16) || ldx % 8 || !aligned(q, 16) || !aligned(out, 16) || !aligned(tensor_scale, 4))
        return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, linear_workspace(m, n, k))) return rc;
    return run_linear(x, ldx, q, scales, block, tensor_scale, m, n, k, out_dtype, out, workspace, (hipStream_t)stream);
}

int64_t nvfp4_matmul_grad_input_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ld) {
    if (const int rc = check_dims(m, n, k)) return rc;
    return grad_workspace(m, n, k, k, ld);
}

int nvfp4_matmul_grad_input(const void* dy, int64_t ld, const uint8_t* q, const uint8_t* scales, int block,
                            const float* tensor_scale, int64_t m, int64_t n, int64_t k, int out_dtype, void* dx,
                            void* workspace, size_t workspace_bytes, void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_nvfp4(m, n, k, block)) return rc;
    if (ld < n || ld > kMaxLd || !grad_launchable(m, n, k, k)) return NVFP4_ERR_SHAPE;
    if (m == 0 || k == 0) return NVFP4_OK;
    if (!dx || !tensor_scale || (n > 0 && (!dy || !q || !scales))) return NVFP4_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(q, 16) || !aligned(dx, 16) || !aligned(tensor_scale, 4)) return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, grad_workspace(m, n, k, k, ld))) return rc;
    return run_grad<kBf16>(dy, ld, q, scales, block, tensor_scale, m, n, k, k, out_dtype, dx, workspace,
                           (hipStream_t)stream);
}

int64_t mxfp4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (const int rc = check_dims(m, n, k)) return rc;
    return mx_workspace(m, n, ceil_div(k, 32));
}

int mxfp4_matmul(const uint8_t* a_q, const uint8_t* a_scales, const uint8_t* b_q, const uint8_t* b_scales, int64_t m,
                 int64_t n, int64_t k, int out_dtype, void* out, void* workspace, size_t workspace_bytes,
                 void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_dims(m, n, k)) return rc;
    if (!mx_launchable(m, n, ceil_div(k, 32))) return NVFP4_ERR_SHAPE;
    if (m == 0 || n == 0) return NVFP4_OK;
    if (!out || (k > 0 && (!a_q || !a_scales || !b_q || !b_scales))) return NVFP4_ERR_NULL;
    if (!aligned(a_q, 16) || !aligned(b_q, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(out, 16))
        return NVFP4_ERR_ALIGN;
    const int64_t blocks = ceil_div(k, 32);
    if (const int rc = check_ws(workspace, workspace_bytes, mx_workspace(m, n, blocks))) return rc;
    return run_mx(a_q, a_scales, b_q, b_scales, m, n, blocks, out_dtype, out, workspace, (hipStream_t)stream);
}

int64_t mxfp4_matmul_grad_input_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ld) {
    if (const int rc = check_dims(m, n, k)) return rc;
    return grad_workspace(m, n, k, up(k, 32), ld);
}

int mxfp4_matmul_grad_input(const void* dy, int64_t ld, const uint8_t* q, const uint8_t* scales, int64_t m, int64_t n,
                            int64_t k, int out_dtype, void* dx, void* workspace, size_t workspace_bytes,
                            void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_dims(m, n, k)) return rc;
    if (ld < n || ld > kMaxLd || !grad_launchable(m, n, k, up(k, 32))) return NVFP4_ERR_SHAPE;
    if (m == 0 || k == 0) return NVFP4_OK;
    if (!dx || (n > 0 && (!dy || !q || !scales))) return NVFP4_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(q, 16) || !aligned(dx, 16)) return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, grad_workspace(m, n, k, up(k, 32), ld))) return rc;
    return run_grad<kMx>(dy, ld, q, scales, 32, nullptr, m, n, k, up(k, 32), out_dtype, dx, workspace,
                         (hipStream_t)stream);
}

}  // extern "C"
