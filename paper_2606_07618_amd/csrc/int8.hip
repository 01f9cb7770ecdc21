// Linear layers in 8-bit integers: rows x = s q with s = max|x| / 127 (the product with binary32's 1/127, as elementary
// operations on tensors divide by a number: at most 0.56 units of its last place off), and the products of two operands so,
//   y[m][n] = s_a[m] s_b[n] sum_k a[m][k] b[n][k],   dx[m][k] = sum_n dy[m][n] s_b[n] b[n][k].
// Integer sums are exact; an output is rounded where the sum becomes a binary32 number, in the product of the scales, in
// their product, and to its type.
#include "dot_product.h"
#include "product_host.h"

namespace {

using namespace product_host;

constexpr int64_t kRowUnit = 16;                          // rows of q hold whole ones, zeros past the width
// 2^14 times as many values stay within 32 bits.
constexpr int64_t kMostInner = ((int64_t)1 << 17) - kRowUnit;

// ---- quantization -----------------------------------------------------------------------------
// One pass: a row stays in registers between its maximum and its quotients, as long as it has at most 8 kKept values a
// thread; what is longer is read again.  A wave a row, or a workgroup where a wave would hold more than half of that.
// From memory, [8192, 4096] bfloat16: 32 us, of which 20 to move: the vector instructions of a quotient and of packing are issued
// 0.6 of the time, and a row waits before it computes.  [777, 14330] binary32: 15 us, 11 to move (three rows a compute unit,
// which all wait first and compute then: 0.2).
constexpr int kQuantThreads = 256, kQuantWaves = kQuantThreads / kLanes, kUnit = 8, kKept = 8;   // units of 8 values

// 8 values from `from`, of which `left` are there: bits of binary32 numbers.
template <bool F32>
struct Eight {
    uint32_t w[F32 ? 8 : 4];
    __device__ __forceinline__ void load(const char* from, int64_t left) {
        if (left >= 8) {
            __builtin_memcpy(w, from, sizeof(w));         // rows begin at any value
            return;
        }
#pragma unroll
        for (int i = 0; i < (F32 ? 8 : 4); ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < left) {
                if constexpr (F32) w[i] = reinterpret_cast<const uint32_t*>(from)[i];
                else w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(from)[i] << i % 2 * 16;
            }
        }
    }
    __device__ __forceinline__ uint32_t bits(int i) const {
        if constexpr (F32) return w[i];
        else return i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16;
    }
};

// The whole number nearest to v / s, ties to the even one, |v| <= about 127 s, both far from binary32's ends.  The
// quotient's estimate is off by one at most; the remainder v - r s is exact, and so is what it says about r.
__device__ __forceinline__ float nearest(float v, float s, float r) {
    const float twice = 2.0f * fmaf(-r, s, v);
    const bool odd = ((int)r & 1) != 0;
    if (twice > s || (twice == s && odd)) r += 1.0f;
    else if (twice < -s || (twice == -s && odd)) r -= 1.0f;
    return fminf(fmaxf(r, -127.0f), 127.0f);
}

// Eight of them, in bytes.  Nearly all quotients lie far from a tie, and their estimates round as they do: only where a
// remainder comes near half a step is each looked at.
template <class E>
__device__ __forceinline__ uint2 nearest8(const E& e, float by, float s, float inverse, float sure) {
    float r[8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = __uint_as_float(e.bits(i)) * by;
        r[i] = rintf(v * inverse);
        most = fmaxf(most, fabsf(fmaf(-r[i], s, v)));
    }
    if (most > sure) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = nearest(__uint_as_float(e.bits(i)) * by, s, r[i]);
    }
    // 1.5 2^23 more, a number's lowest byte is the whole number's
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(r[4 * h + i] + 12582912.0f);
        w[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0C0C0400u), __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u), 0x05040100u);
    }
    return make_uint2(w[0], w[1]);
}

template <bool F32, bool WAVE>
__global__ __launch_bounds__(kQuantThreads) void quant_kernel(const char* __restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                              int8_t* __restrict__ q, float* __restrict__ scales) {
    __shared__ uint32_t tops[kQuantWaves];
    constexpr int kSpan = (WAVE ? kLanes : kQuantThreads) * kUnit;      // values that a row's threads cover
    constexpr int kSize = F32 ? 4 : 2;
    const int tid = threadIdx.x, lane = tid % kLanes, wave = tid / kLanes;
    const int64_t row = WAVE ? (int64_t)blockIdx.x * kQuantWaves + wave : blockIdx.x;
    if (WAVE && row >= rows) return;
    const char* from = x + row * ld * kSize;
    const int64_t first = (WAVE ? lane : tid) * kUnit, q_ld = (cols + kRowUnit - 1) / kRowUnit * kRowUnit;
    Eight<F32> kept[kKept];
    uint32_t top = 0;
    auto join = [&](const Eight<F32>& e) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = e.bits(i) & 0x7FFFFFFFu;   // magnitudes order as their bits do, infinities and NaN on top
            top = a > top ? a : top;
        }
    };
#pragma unroll
    for (int u = 0; u < kKept; ++u) {
        const int64_t at = first + (int64_t)u * kSpan;
        kept[u].load(from + at * kSize, cols - at);
        if (at >= cols) continue;
        join(kept[u]);
    }
    for (int64_t at = first + (int64_t)kKept * kSpan; at < cols; at += kSpan) {
        Eight<F32> e;
        e.load(from + at * kSize, cols - at);
        join(e);
    }
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) {
        const uint32_t o = __shfl_xor(top, d);
        top = o > top ? o : top;
    }
    if constexpr (!WAVE) {
        if (lane == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantWaves; ++w) top = tops[w] > top ? tops[w] : top;
    }
    const bool finite = top < 0x7F800000u;
    const float s = __uint_as_float(top) * 0x1.020408p-7f;
    if ((WAVE ? lane : tid) == 0) scales[row] = finite ? s : __uint_as_float(0x7FC00000u);
    // small scales and their rows times 2^64, exactly, so that neither the reciprocal nor a remainder leaves the range
    const float by = s < 0x1p-100f ? 0x1p64f : 1.0f, sb = s * by;
    const float inverse = finite && s > 0.0f ? 1.0f / sb : 0.0f;
    // rows of subnormal scales, whose quotients may pass 127, are looked at one by one
    const float sure = s < 0x1p-120f ? -1.0f : 0.4999f * sb;
    auto store = [&](const Eight<F32>& e, int64_t at) {
        *reinterpret_cast<uint2*>(q + row * q_ld + at) = inverse > 0.0f ? nearest8(e, by, sb, inverse, sure) : make_uint2(0, 0);
    };
#pragma unroll
    for (int u = 0; u < kKept; ++u) {
        const int64_t at = first + (int64_t)u * kSpan;
        if (at < q_ld) store(kept[u], at);                // past the width: zeros
    }
    for (int64_t at = first + (int64_t)kKept * kSpan; at < q_ld; at += kSpan) {
        Eight<F32> e;
        e.load(from + at * kSize, cols - at);
        store(e, at);
    }
}

constexpr int64_t kWaveCols = kLanes * kUnit * kKept / 2;

int64_t quant_groups(int64_t rows, int64_t cols) { return cols <= kWaveCols ? ceil_div(rows, kQuantWaves) : rows; }

// ---- one to four rows -------------------------------------------------------------------------
// As the NVFP4 products of so few rows: lanes along the contraction, 16 values each, eight weight rows on their way at
// once, four products an instruction.  One row, [14336, 4096], from memory: 12 us, 4.9 TB/s.
constexpr int kDotSpan = kLanes * 16, kDotN = 8, kDotWaves = dot_product::kWaves;

struct DotArgs {
    const char *a, *b;
    const float *scale_m, *scale_n;
    int64_t n, k;                                // k: bytes of a row
    int along;                                   // waves of a workgroup along the contraction
    void* out;
    int out_f32;
};

__device__ __forceinline__ int fold32(int a, int b) {
    const dot_product::u32x2 r = __builtin_amdgcn_permlane32_swap((uint32_t)a, (uint32_t)b, false, false);
    return (int)(r[0] + r[1]);
}
__device__ __forceinline__ int fold16(int a, int b) {
    const dot_product::u32x2 r = __builtin_amdgcn_permlane16_swap((uint32_t)a, (uint32_t)b, false, false);
    return (int)(r[0] + r[1]);
}
template <int CTRL>
__device__ __forceinline__ int add_dpp(int v) { return v + __builtin_amdgcn_mov_dpp(v, CTRL, 0xF, 0xF, true); }
// The sum over each row of 16 lanes, in all of them.
__device__ __forceinline__ int sum16(int v) {
    v = add_dpp<0xB1>(v);
    v = add_dpp<0x4E>(v);
    v = add_dpp<0x141>(v);
    return add_dpp<0x140>(v);
}

template <int M>
__global__ __launch_bounds__(kDotWaves * kLanes) void int8_dot_kernel(DotArgs p) {
    __shared__ int sums[kDotWaves][M][kDotN];
    const int tid = threadIdx.x, lane = tid % kLanes;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int along = p.along, part = wave % along, group = wave / along, rows = kDotN * (kDotWaves / along);
    const int64_t n0 = (int64_t)blockIdx.x * rows + group * kDotN, left = p.n - n0;
    const uint32_t k = (uint32_t)p.k;
    const __amdgpu_buffer_rsrc_t rb = window(p.b + n0 * p.k), ra = window(p.a);
    int acc[M][kDotN];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < kDotN; ++r) acc[m][r] = 0;
    for (uint32_t at = (uint32_t)part * kDotSpan; at < k; at += (uint32_t)along * kDotSpan) {
        const uint32_t v = at + lane * 16;
        i32x4 x[M], w[kDotN];
#pragma unroll
        for (int r = 0; r < kDotN; ++r) w[r] = load16(rb, r < left && v < k ? r * k + v : kOutside);
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = load16(ra, v < k ? m * k + v : kOutside);
#pragma unroll
        for (int r = 0; r < kDotN; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[m][r] = __builtin_amdgcn_sdot4(w[r][j], x[m][j], acc[m][r], false);
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
        static_assert(kDotN == 8, "two folds and a pair");
        const int a = sum16(fold16(fold32(acc[m][0], acc[m][2]), fold32(acc[m][1], acc[m][3])));
        const int b = sum16(fold16(fold32(acc[m][4], acc[m][6]), fold32(acc[m][5], acc[m][7])));
        if (lane % 16 == 0) {
            sums[wave][m][lane / 16] = a;
            sums[wave][m][4 + lane / 16] = b;
        }
    }
    __syncthreads();
    if (tid >= M * rows) return;
    const int r = tid % kDotN, m = tid / kDotN % M, of = tid / (kDotN * M);
    int v = 0;
    for (int a = 0; a < along; ++a) v += sums[of * along + a][m][r];
    const int64_t n = (int64_t)blockIdx.x * rows + of * kDotN + r;
    if (n >= p.n) return;
    const float y = scaled(v, p.scale_n[n], p.scale_m[m]);
    if (p.out_f32) static_cast<float*>(p.out)[m * p.n + n] = y;
    else static_cast<uint16_t*>(p.out)[m * p.n + n] = (uint16_t)pack_bf16(y, y);
}

template <int M>
void launch_dot(const DotArgs& p, hipStream_t stream) {
    const int rows = kDotN * (kDotWaves / p.along);
    hipLaunchKernelGGL((int8_dot_kernel<M>), dim3((unsigned)ceil_div(p.n, rows)), dim3(kDotWaves * kLanes), 0, stream, p);
}

// ---- tiles ------------------------------------------------------------------------------------
// The tiled product of the other operands: a step's 128 bytes of a row are 128 values.  [8192, 4096] x [14336, 4096]: 380 us
// on one card, 400 from memory on another, 2.5 and 2.4 POP/s (a library's [8192, 8192] x [8192, 8192] of integers: 2.1).

// Sums of parts of the contraction, in 32-bit integers as a whole sum is: a workgroup for kJoinColumns outputs of a row.
// Rows of parts hold whole fours, which a tile stores at once.
constexpr int kJoinColumns = kJoinThreads * 4;

__global__ __launch_bounds__(kJoinThreads) void int8_join_kernel(const int* __restrict__ part, int parts, int64_t m, int64_t n, int64_t ld, uint32_t pieces,
                                                                 const float* __restrict__ scale_m, const float* __restrict__ scale_n,
                                                                 void* __restrict__ out, int f32) {
    const int64_t row = blockIdx.x / pieces, first = (int64_t)(blockIdx.x % pieces) * kJoinColumns + threadIdx.x;
    const float s = scale_m[row];
    int v[4] = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const int* from = part + (p * m + row) * ld + first;
#pragma unroll
        for (int i = 0; i < 4; ++i) if (first + i * kJoinThreads < n) v[i] += from[i * kJoinThreads];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t c = first + i * kJoinThreads;
        if (c >= n) break;
        const float y = scaled(v[i], scale_n[c], s);
        if (f32) static_cast<float*>(out)[row * n + c] = y;
        else static_cast<uint16_t*>(out)[row * n + c] = (uint16_t)pack_bf16(y, y);
    }
}

int64_t join_groups(int64_t m, int64_t n) { return m * ceil_div(n, kJoinColumns); }

int64_t int8_workspace(int64_t m, int64_t n, int64_t k) {
    if (m <= kDotRows) return 0;
    const int parts = plan_product<kInt8, kSums>(m, n, up(k, kRowUnit)).parts;
    return parts > 1 ? up(parts * m * up(n, 4) * 4, 256) : 0;
}

bool int8_launchable(int64_t m, int64_t n, int64_t k) {
    return m <= kDotRows || (product_launchable<kInt8>(m, n, up(k, kRowUnit)) && launchable(join_groups(m, n), kJoinThreads));
}

int run_int8(const int8_t* a, const float* a_scales, const int8_t* b, const float* b_scales, int64_t m, int64_t n, int64_t k,
             int out_dtype, void* out, void* ws, hipStream_t stream) {
    const int f32 = out_dtype == NVFP4_IN_F32;
    if (m <= kDotRows) {
        DotArgs t = {reinterpret_cast<const char*>(a), reinterpret_cast<const char*>(b), a_scales, b_scales, n, k,
                     dot_product::waves_along(k, kDotSpan), out, f32};
        switch (m) {
            case 1: launch_dot<1>(t, stream); break;
            case 2: launch_dot<2>(t, stream); break;
            case 3: launch_dot<3>(t, stream); break;
            default: launch_dot<4>(t, stream);
        }
        return launched();
    }
    Args p = {};
    p.a.p = reinterpret_cast<const char*>(a), p.a.ld = k;
    p.b.p = reinterpret_cast<const char*>(b), p.b.ld = k;
    p.m = m, p.n = n, p.inner = k, p.out = out, p.out_ld = n, p.out_f32 = f32, p.scale_m = a_scales, p.scale_n = b_scales;
    const Plan plan = plan_product<kInt8, kSums>(m, n, k);
    p.parts = plan.parts;
    if (plan.parts == 1) return launch_product<kInt8, kSums>(p, plan.tile, stream);
    p.out = ws, p.out_ld = up(n, 4);
    if (const int rc = launch_product<kInt8, kPartial>(p, plan.tile, stream)) return rc;
    hipLaunchKernelGGL(int8_join_kernel, dim3((unsigned)join_groups(m, n)), dim3(kJoinThreads), 0, stream,
                       static_cast<const int*>(ws), plan.parts, m, n, up(n, 4), (uint32_t)ceil_div(n, kJoinColumns), a_scales, b_scales, out, f32);
    return launched();
}

// ---- the gradient with respect to the rows ------------------------------------------------------
// The scales run along the contraction here, so the weights are expanded to bfloat16, rows turned.  s q has up to 31
// significant bits.  For a bfloat16 gradient it is rounded to 8, which takes the gradient's relative error from 0.0017, its
// own rounding, to 0.0023 or 0.0024 ([4096, 14336] x [14336, 4096]: 375 us; 1210 with whole weights).  A binary32 gradient is for
// those who need more: binary32's s q is three bfloat16 numbers, each the largest below what those before it leave (exact from
// 2^-109 on), and three products, one on top of the other, through one buffer of weights.  Below, not up to: none of the three is
// zero then, and an infinite dy gives an infinity as it does with the weight itself.
enum Term { kRounded, kFirst, kSecond, kThird };

template <Term TERM>
__device__ __forceinline__ float term_of(float w) {
    if constexpr (TERM == kRounded) return w;                 // by the conversion
    const auto below = [](float v) {                          // in magnitude
        const uint32_t bits = __float_as_uint(v), size = bits & 0x7FFFFFFFu;
        return __uint_as_float((bits & 0x80000000u) | (size == 0 ? 0 : (size - 1) & 0xFFFF0000u));
    };
    if (!(fabsf(w) < __builtin_inff())) return w;             // an infinity or a NaN three times
    const float first = below(w), rest = w - first, second = below(rest);
    return TERM == kFirst ? first : TERM == kSecond ? second : rest - second;
}

constexpr int kTurnThreads = 256, kTurnN = 64, kTurnK = 128;

template <Term TERM>
__global__ __launch_bounds__(kTurnThreads) void int8_turned_kernel(const int8_t* __restrict__ q, const float* __restrict__ scales,
                                                                   int64_t n, uint32_t k, uint32_t tiles_k, int64_t ld,
                                                                   uint16_t* __restrict__ out) {
    // a row is two words longer than its values, so that a wave's writes meet in few banks
    __shared__ uint32_t tile[kTurnK][kTurnN / 2 + 1];
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_k) * kTurnN;
    const uint32_t k0 = blockIdx.x % tiles_k * kTurnK;
    const int row = threadIdx.x / 4, part = threadIdx.x % 4;             // 16 values of a weight row, 64 apart
    const bool row_in = n0 + row < n;
    const float s = row_in ? scales[n0 + row] : 0.0f;
    constexpr int kPieces = kTurnK / 64;
    i32x4 w[kPieces];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        const uint32_t at = k0 + p * 64 + part * 16;                     // k is a multiple of 16
        w[p] = row_in && at < k ? *reinterpret_cast<const i32x4*>(q + (n0 + row) * k + at) : i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const int a = (int)(int8_t)(w[p][j / 4] >> j % 4 * 8), b = (int)(int8_t)(w[p][j / 4] >> (j % 4 + 1) * 8);
            const uint32_t v = pack_bf16(term_of<TERM>((float)a * s), term_of<TERM>((float)b * s));
            reinterpret_cast<uint16_t*>(tile[p * 64 + part * 16 + j])[row] = (uint16_t)v;
            reinterpret_cast<uint16_t*>(tile[p * 64 + part * 16 + j + 1])[row] = (uint16_t)(v >> 16);
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurnK * kTurnN / 8 / kTurnThreads; ++i) {
        const int c = i * kTurnThreads + threadIdx.x, r = c / (kTurnN / 8), chunk = c % (kTurnN / 8);
        if (k0 + r < k && n0 + chunk * 8 < ld)
            *reinterpret_cast<uint4*>(out + (int64_t)(k0 + r) * ld + n0 + chunk * 8) =
                make_uint4(tile[r][chunk * 4], tile[r][chunk * 4 + 1], tile[r][chunk * 4 + 2], tile[r][chunk * 4 + 3]);
    }
}

int64_t turned_groups(int64_t n, int64_t k) { return ceil_div(n, kTurnN) * ceil_div(up(k, kRowUnit), kTurnK); }

int64_t int8_grad_workspace(int64_t m, int64_t n, int64_t k, int64_t ld) {
    Carver c{nullptr};
    c.take(up(k, kRowUnit) * packed_ld(n) * 2);
    if (needs_pack(n, ld)) c.take(m * packed_ld(n) * 2);
    return c.at + parts_bytes<kBf16>(m, k, n);
}

// One product on a term of the weights, which `w` holds until it is done.
template <Term TERM, Out OUT>
int grad_product(const int8_t* q, const float* scales, int64_t n, int64_t k, void* w, const Args& p, float* partial, hipStream_t stream) {
    const int64_t row = up(k, kRowUnit);
    if (n > 0) {
        hipLaunchKernelGGL((int8_turned_kernel<TERM>), dim3((unsigned)turned_groups(n, k)), dim3(kTurnThreads), 0, stream, q, scales, n,
                           (uint32_t)row, (uint32_t)ceil_div(row, kTurnK), packed_ld(n), static_cast<uint16_t*>(w));
        if (const int rc = launched()) return rc;
    }
    return run_sums<kBf16, OUT>(p, partial, stream);
}

int run_int8_grad(const void* dy, int64_t ld, const int8_t* q, const float* scales, int64_t m, int64_t n, int64_t k, int out_dtype,
                  void* out, void* ws, hipStream_t stream) {
    Carver c{static_cast<char*>(ws)};
    void* w = c.take(up(k, kRowUnit) * packed_ld(n) * 2);
    if (needs_pack(n, ld)) {
        void* packed = c.take(m * packed_ld(n) * 2);
        if (const int rc = pack_bf16_rows(dy, m, n, ld, packed, stream)) return rc;
        dy = packed, ld = packed_ld(n);
    }
    Args p = {};
    p.a.p = static_cast<const char*>(dy), p.a.ld = ld * 2;
    p.b.p = static_cast<const char*>(w), p.b.ld = packed_ld(n) * 2;
    p.m = m, p.n = k, p.inner = n, p.out = out, p.out_ld = k, p.out_f32 = out_dtype == NVFP4_IN_F32;
    float* partial = static_cast<float*>(c.take(0));
    if (!p.out_f32) return grad_product<kRounded, kSums>(q, scales, n, k, w, p, partial, stream);
    // the smallest first: with the second it adds up to all that the first leaves, and that with the first to the weight
    if (const int rc = grad_product<kThird, kSums>(q, scales, n, k, w, p, partial, stream)) return rc;
    if (const int rc = grad_product<kSecond, kAdded>(q, scales, n, k, w, p, partial, stream)) return rc;
    return grad_product<kFirst, kAdded>(q, scales, n, k, w, p, partial, stream);
}

int check_int8(int64_t m, int64_t n, int64_t k) {
    if (const int rc = check_dims(m, n, k)) return rc;
    return k > kMostInner ? NVFP4_ERR_SHAPE : NVFP4_OK;
}

bool valid_out(int dtype) { return dtype == NVFP4_IN_F32 || dtype == NVFP4_IN_BF16; }

}  // namespace

extern "C" {

int int8_quant(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* q, float* scales, void* stream) {
    if (!valid_out(dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_int8(rows, 0, cols)) return rc;
    if (ldx < cols || ldx > kMaxLd || !launchable(quant_groups(rows, cols), kQuantThreads)) return NVFP4_ERR_SHAPE;
    if (rows == 0) return NVFP4_OK;
    if (!scales || (cols > 0 && (!x || !q))) return NVFP4_ERR_NULL;
    const bool f32 = dtype == NVFP4_IN_F32, wave = cols <= kWaveCols;
    if (!aligned(x, f32 ? 4 : 2) || !aligned(q, 16) || !aligned(scales, 4)) return NVFP4_ERR_ALIGN;
    auto kernel = f32 ? (wave ? quant_kernel<true, true> : quant_kernel<true, false>)
                      : (wave ? quant_kernel<false, true> : quant_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)quant_groups(rows, cols)), dim3(kQuantThreads), 0, (hipStream_t)stream,
                       static_cast<const char*>(x), rows, cols, ldx, q, scales);
    return launched();
}

int64_t int8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (const int rc = check_int8(m, n, k)) return rc;
    return int8_workspace(m, n, k);
}

int int8_matmul(const int8_t* a_q, const float* a_scales, const int8_t* b_q, const float* b_scales, int64_t m, int64_t n,
                int64_t k, int out_dtype, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_int8(m, n, k)) return rc;
    if (!int8_launchable(m, n, k)) return NVFP4_ERR_SHAPE;
    if (m == 0 || n == 0) return NVFP4_OK;
    if (!out || !a_scales || !b_scales || (k > 0 && (!a_q || !b_q))) return NVFP4_ERR_NULL;
    if (!aligned(a_q, 16) || !aligned(b_q, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(out, 16))
        return NVFP4_ERR_ALIGN;
    if (const int rc = check_workspace(workspace, workspace_bytes, int8_workspace(m, n, k))) return rc;
    return run_int8(a_q, a_scales, b_q, b_scales, m, n, up(k, kRowUnit), out_dtype, out, workspace, (hipStream_t)stream);
}

int64_t int8_matmul_grad_input_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ld) {
    if (const int rc = check_int8(m, n, k)) return rc;
    return int8_grad_workspace(m, n, k, ld);
}

int int8_matmul_grad_input(const void* dy, int64_t ld, const int8_t* q, const float* scales, int64_t m, int64_t n, int64_t k,
                           int out_dtype, void* dx, void* workspace, size_t workspace_bytes, void* stream) {
    if (!valid_out(out_dtype)) return NVFP4_ERR_DTYPE;
    if (const int rc = check_int8(m, n, k)) return rc;
    if (ld < n || ld > kMaxLd || !launchable(turned_groups(n, k), kTurnThreads) || !product_launchable<kBf16>(m, k, n))
        return NVFP4_ERR_SHAPE;
    if (m == 0 || k == 0) return NVFP4_OK;
    if (!dx || (n > 0 && (!dy || !q || !scales))) return NVFP4_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(q, 16) || !aligned(scales, 4) || !aligned(dx, 16)) return NVFP4_ERR_ALIGN;
    if (const int rc = check_workspace(workspace, workspace_bytes, int8_grad_workspace(m, n, k, ld))) return rc;
    return run_int8_grad(dy, ld, q, scales, m, n, k, out_dtype, dx, workspace, (hipStream_t)stream);
}

}  // extern "C"
