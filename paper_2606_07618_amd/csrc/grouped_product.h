// Products of rows sorted by group (the tokens of each expert) with the NVFP4 weights of their own group.  Where a
// group's rows begin is known on the device alone, so a workgroup finds its rows itself: tiles are numbered through all
// groups, and each wave sums the groups' tile counts up to its own number.
//
//   y[i][n]  = S_e sum_k x[i][k] (q s)_e[n][k]      weights as they lie: the contraction runs along their rows
//   dx[i][k] = S_e sum_n dy[i][n] (q s)_e[n][k]     turned: it runs down their rows
//
// A weight q s has six significant bits and is exact in bfloat16, the type of the rows; sums are binary32.
#pragma once

#include "stream_product.h"

namespace grouped_product {

using namespace tile_product;
using stream_product::expand8;

struct Args {
    const char* x;                               // [rows, ld bytes]
    int64_t ld, rows;
    const int* offsets;                          // [experts + 1]
    int experts, shift;                          // 1 << shift: values of a block
    const char* q;                               // [experts, n, k / 2]
    const uint8_t* scales;                       // [experts, n, k >> shift]
    const float* S;                              // [experts]
    int64_t n, k;
    int64_t inner, outer;                        // of the product: k, n, or n, k where turned
    int64_t tiles_n;
    void* out;                                   // [rows, outer]
    int out_f32, clear;                          // clear: rows of no group become zero
};

// Where a tile lies: its expert, its rows first .. first + left - 1 (left: to the group's end).  expert < 0: none; then
// the groups' rows are begin .. end - 1, and `index` counts on from the last tile.
struct Place { int expert; int64_t first, left, begin, end, index; };

__device__ __forceinline__ int at_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Offsets are taken within 0 .. rows and never descend: what does not fit makes a group shorter or empty.
__device__ __forceinline__ Place place_of(const Args& p, int64_t index, int height, int lane) {
    const int rows = (int)p.rows;
    auto within = [&](int v) { return v < 0 ? 0 : v > rows ? rows : v; };
    int before = within(p.offsets[0]);
    const int begin = before;
    for (int base = 0; base < p.experts; base += kLanes) {
        const int e = base + lane;
        int end = e < p.experts ? within(p.offsets[e + 1]) : 0;
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) {
            const int v = __shfl_up(end, d);
            if (lane >= d && v > end) end = v;
        }
        if (end < before) end = before;
        int start = __shfl_up(end, 1);
        if (lane == 0) start = before;
        int64_t tiles = (end - start + (int64_t)height - 1) / height;
        int64_t upto = tiles;
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) {
            const int64_t v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const uint64_t mine = __ballot(index < upto);
        if (mine) {
            const int l = __builtin_ctzll(mine);
            const int64_t skipped = at_lane((int)(upto - tiles), l);
            const int s = at_lane(start, l), t = at_lane(end, l);
            const int64_t first = s + (index - skipped) * height;
            return {base + l, first, t - first, 0, 0, 0};
        }
        index -= at_lane((int)upto, kLanes - 1);
        before = at_lane(end, kLanes - 1);
    }
    return {-1, 0, 0, begin, before, index};
}

// Rows of no group: the workgroups that have no tile share them out.
__device__ __forceinline__ void clear_rows(const Args& p, const Place& t, int64_t n0, int64_t width, int64_t sharers, int tid,
                                           int threads) {
    if (!p.clear) return;
    const int64_t end = n0 + width < p.outer ? n0 + width : p.outer;
    for (int64_t i = t.index; i < t.begin + (p.rows - t.end); i += sharers) {
        const int64_t m = i < t.begin ? i : t.end + (i - t.begin);
        for (int64_t n = n0 + tid; n < end; n += threads) {
            if (p.out_f32) static_cast<float*>(p.out)[m * p.outer + n] = 0.0f;
            else static_cast<uint16_t*>(p.out)[m * p.outer + n] = 0;
        }
    }
}

// Row tile and columns from a workgroup's number: an XCD gets a run of the sequence, which walks kDeep row tiles at a
// time, so that what it works on at one time shares rows and weights in its L2.
constexpr int kDeep = 4;
struct Work { int64_t index, n; };
__device__ __forceinline__ Work work_of(int64_t id, int64_t count, int64_t tiles_n) {
    const int64_t xcd = id % kXcds, each = count / kXcds, rest = count % kXcds, tiles_m = count / tiles_n;
    const int64_t seq = xcd * each + (xcd < rest ? xcd : rest) + id / kXcds;
    const int64_t first = seq / (kDeep * tiles_n) * kDeep, height = tiles_m - first < kDeep ? tiles_m - first : kDeep;
    const int64_t in = seq % (kDeep * tiles_n);
    return {first + in % height, in / height};
}

// ---- few rows a group ---------------------------------------------------------------------------
// Reading the weights is all there is to do.  A workgroup owns 16 R weight rows and up to 16 C rows of one group; its waves
// take turns along the contraction, 256 values (whole lines of the weights) each, loaded straight into the registers of
// the matrix instructions, and one exchange through LDS adds their sums in a fixed order.
constexpr int kFewWaves = 8, kFewGroup = 256;

// How a lane gets the scales of its 32 values: two, one, or two of which the second may lie past the row (and so may half
// of the values).
enum Scales { kPair, kOne, kOdd };

template <int R, int C, Scales SCALES>
__global__ __launch_bounds__(kFewWaves * kLanes) void few_kernel(Args p) {
    __shared__ f32x4 sums[kFewWaves][R * C][kLanes];
    const int tid = threadIdx.x, lane = tid % kLanes, g = lane / 16, i16 = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const Work work = work_of(blockIdx.x, gridDim.x, p.tiles_n);
    const int64_t n0 = work.n * (16 * R);
    const Place t = place_of(p, work.index, 16 * C, lane);
    if (t.expert < 0) return clear_rows(p, t, n0, 16 * R, gridDim.x / p.tiles_n - (work.index - t.index), tid, kFewWaves * kLanes);

    const uint32_t k = (uint32_t)p.k, q_ld = k / 2, s_ld = k >> p.shift;
    const int64_t row0 = t.expert * p.n + n0;
    const __amdgpu_buffer_rsrc_t rq = window(p.q + row0 * q_ld), rs = window(p.scales + row0 * s_ld), rx = window(p.x + t.first * p.ld);
    bool row_in[R], x_in[C];
#pragma unroll
    for (int r = 0; r < R; ++r) row_in[r] = n0 + r * 16 + i16 < p.n;
#pragma unroll
    for (int c = 0; c < C; ++c) x_in[c] = c * 16 + i16 < t.left;
    f32x4 acc[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) acc[r][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (uint32_t at = (uint32_t)wave * kFewGroup; at < k; at += kFewWaves * kFewGroup) {
        i32x4 w[2][R];
        uint32_t s[2][R];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t v = at + h * 128 + g * 32;
            const bool in0 = v < k, in1 = SCALES == kOdd ? v + 16 < k : in0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint32_t row = r * 16 + i16, q_at = row * q_ld + v / 2, s_at = row * s_ld + (v >> p.shift);
                if constexpr (SCALES == kOdd) {
                    const i32x2 lo = load8(rq, row_in[r] && in0 ? q_at : kOutside), hi = load8(rq, row_in[r] && in1 ? q_at + 8 : kOutside);
                    w[h][r] = i32x4{lo[0], lo[1], hi[0], hi[1]};
                    s[h][r] = load1(rs, row_in[r] && in0 ? s_at : kOutside) | load1(rs, row_in[r] && in1 ? s_at + 1 : kOutside) << 8;
                } else {
                    w[h][r] = load16(rq, row_in[r] && in0 ? q_at : kOutside);
                    if constexpr (SCALES == kPair)
                        s[h][r] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(row_in[r] && in0 ? s_at : kOutside), 0, 0);
                    else s[h][r] = load1(rs, row_in[r] && in0 ? s_at : kOutside);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t v = at + h * 128 + g * 32;
            const bool in0 = v < k, in1 = SCALES == kOdd ? v + 16 < k : in0;
            i32x4 x[C][4];
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[c][j] = load16(rx, x_in[c] && (j < 2 ? in0 : in1) ? (uint32_t)(c * 16 + i16) * (uint32_t)p.ld + v * 2 + j * 16 : kOutside);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f0 = e4m3_f32(s[h][r]), f1 = SCALES == kOne ? f0 : e4m3_f32(s[h][r] >> 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 wv = expand8((uint32_t)w[h][r][j], j < 2 ? f0 : f1);
#pragma unroll
                    for (int c = 0; c < C; ++c)
                        acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, x[c][j]), acc[r][c], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) sums[wave][r * C + c][lane] = acc[r][c];
    __syncthreads();
    const float S = p.S[t.expert];
    for (int f = wave; f < R * C; f += kFewWaves) {
        f32x4 v = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) v += sums[w][f][lane];
        // a lane holds outputs n .. n + 3 of row i16
        const int64_t n = n0 + f / C * 16 + g * 4, row = f % C * 16 + i16;
        if (row < t.left) store4(p.out, p.out_f32, (t.first + row) * p.outer + n, p.outer - n, p.outer % 4 == 0, v * S);
    }
}

// ---- tiles --------------------------------------------------------------------------------------
// Weights are expanded by the threads that load them, once for a tile's rows, on their way into LDS, where they lie as
// bfloat16 rows along the contraction, turned or not: turning costs nothing, as the pairs that share a register are put
// together from single values anyway.  The rows of the other operand go from memory straight into LDS.  A step of the
// contraction is 64 values; registers hold the weights of the next two steps, LDS the rows and weights of two.
// A group's last tile computes as many rows as it needs, in halves.
constexpr int kSteps = 2;                        // in LDS

// A row's chunks of 16 bytes exchanged by the row: reads take one chunk of 16 neighbouring rows, turned writes one of
// rows 8 apart.
__device__ __forceinline__ int exchange(int row) { return ((row >> 1) ^ (row >> 4)) & 7; }

template <int M_, int WN_, int LEAST_>
struct Tile {
    static constexpr int M = M_, WM = 2, WN = WN_, N = WN_ * 64, kThreads = WM * WN_ * kLanes;
    static constexpr int kMost = M_ / 32, kLeast = LEAST_ / 32;      // a wave's fragments of rows
};

template <class T, bool TURNED, Scales SCALES>
struct Weights {
    // As they lie: 32 values of a row.  Turned: 8 columns of four rows.
    static constexpr int kLoads = TURNED ? 8 : SCALES == kOdd ? 4 : 2;
    i32x4 v;
    uint32_t s[TURNED ? 4 : 1];

    // s0: the step's first value of the contraction
    __device__ __forceinline__ void load(const Args& p, __amdgpu_buffer_rsrc_t rq, __amdgpu_buffer_rsrc_t rs, int64_t n0, int64_t s0, int tid) {
        const uint32_t q_ld = (uint32_t)(p.k / 2), s_ld = (uint32_t)(p.k >> p.shift);
        if constexpr (TURNED) {
            const int column = tid % (T::N / 8) * 8, row = tid / (T::N / 8) * 4;
            const bool in = n0 + column < p.k;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool here = in && s0 + row + r < p.n;
                const uint32_t at = (uint32_t)(row + r);
                v[r] = __builtin_amdgcn_raw_buffer_load_b32(rq, (int)(here ? at * q_ld + (uint32_t)column / 2 : kOutside), 0, 0);
                s[r] = load1(rs, here ? at * s_ld + (((uint32_t)n0 + column) >> p.shift) : kOutside);
            }
        } else {
            const int row = tid / 2;
            const uint32_t at = (uint32_t)s0 + tid % 2 * 32, k = (uint32_t)p.k;
            const bool here = n0 + row < p.n, in0 = here && at < k;
            const uint32_t q_at = (uint32_t)row * q_ld + at / 2, s_at = (uint32_t)row * s_ld + (at >> p.shift);
            if constexpr (SCALES == kOdd) {
                const bool in1 = here && at + 16 < k;
                const i32x2 lo = load8(rq, in0 ? q_at : kOutside), hi = load8(rq, in1 ? q_at + 8 : kOutside);
                v = i32x4{lo[0], lo[1], hi[0], hi[1]};
                s[0] = load1(rs, in0 ? s_at : kOutside) | load1(rs, in1 ? s_at + 1 : kOutside) << 8;
            } else {
                v = load16(rq, in0 ? q_at : kOutside);
                if constexpr (SCALES == kPair) s[0] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(in0 ? s_at : kOutside), 0, 0);
                else s[0] = load1(rs, in0 ? s_at : kOutside);
            }
        }
    }

    // Part H of 2.
    template <int H>
    __device__ __forceinline__ void store(char* lds, int tid) const {
        if constexpr (TURNED) {
            const int column = tid % (T::N / 8) * 8, row = tid / (T::N / 8) * 4;
            float f[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) f[r] = e4m3_f32(s[r]);
            const auto pair = [&](int r, auto c) {
                return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[r], 1.0f, decltype(c)::value) * f[r];
            };
            const auto columns = [&](auto c) {           // two of them
                const f32x2 a = pair(0, c), b = pair(1, c), d = pair(2, c), e = pair(3, c);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int to = column + 2 * decltype(c)::value + j;
                    // the upper halves of the products hold all of them
                    const uint2 w = {__builtin_amdgcn_perm(__float_as_uint(b[j]), __float_as_uint(a[j]), 0x07060302u),
                                     __builtin_amdgcn_perm(__float_as_uint(e[j]), __float_as_uint(d[j]), 0x07060302u)};
                    *reinterpret_cast<uint2*>(lds + to * kStepBytes + ((row / 8) ^ exchange(to)) * kChunk + row % 8 * 2) = w;
                }
            };
            columns(Const<2 * H>{}), columns(Const<2 * H + 1>{});
        } else {
            const int row = tid / 2, chunk = tid % 2 * 4;
            const float f = e4m3_f32(SCALES == kOne || H == 0 ? s[0] : s[0] >> 8);
#pragma unroll
            for (int j = 2 * H; j < 2 * H + 2; ++j)
                *reinterpret_cast<bf16x8*>(lds + row * kStepBytes + ((chunk + j) ^ exchange(row)) * kChunk) = expand8((uint32_t)v[j], f);
        }
    }
};

// The product of one tile, MF fragments of 16 rows a wave.
template <class T, bool TURNED, Scales SCALES, int MF>
__device__ __forceinline__ void product(const Args& p, const Place& t, int64_t n0, char (*lds)[(T::M + T::N) * kStepBytes], int tid) {
    constexpr int NF = 4, kRows = MF * 32;
    using A = Side<kRows, T::kThreads, false>;
    using B = Weights<T, TURNED, SCALES>;
    const int lane = tid % kLanes, wave = __builtin_amdgcn_readfirstlane(tid / kLanes), wm = wave / T::WN, wn = wave % T::WN;
    A sa;
    sa.init(t.left, p.ld, tid);
    const char* a0 = p.x + t.first * p.ld;
    const int64_t row_bytes = p.inner * 2, q_ld = p.k / 2, s_ld = p.k >> p.shift;
    const int64_t w_row = t.expert * p.n + (TURNED ? 0 : n0);
    auto fetch_a = [&](int64_t s, int slot) {
        sa.load(a0 + s * kStepBytes, nullptr, lds[slot], row_bytes - s * kStepBytes, tid, wave);
    };
    auto fetch_b = [&](int64_t s, B& b) {
        // turned, the window moves down the rows; else a tile's rows stay within it
        const int64_t row = w_row + (TURNED ? s * 64 : 0);
        b.load(p, window(p.q + row * q_ld + (TURNED ? n0 / 2 : 0)), window(p.scales + row * s_ld), n0, s * 64, tid);
    };
    auto a_row = [&](int i) { return wm * (MF * 16) + i * 16; };
    auto b_row = [&](int j) { return wn * 64 + j * 16; };
    auto read_b = [&](const char* b, int j, int h) {
        const int row = b_row(j) + lane % 16, chunk = 4 * h + lane / 16;
        return *reinterpret_cast<const i32x4*>(b + row * kStepBytes + ((chunk ^ exchange(row)) * kChunk));
    };

    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int64_t steps = (p.inner + 63) / 64;
    B b[2];
    auto in_order = [] { asm volatile("" ::: "memory"); };   // the waits count on it
    auto step = [&](int64_t s, auto dc) {
        constexpr int d = decltype(dc)::value;
        const char *la = lds[d], *lb = lds[d] + T::M * kStepBytes;
        char* next = lds[1 - d] + T::M * kStepBytes;
        // the next step's weights, then those of the step two behind it
        b[1 - d].template store<0>(next, tid);
        b[1 - d].template store<1>(next, tid);
        in_order();
        fetch_b(s + 3, b[1 - d]);
        in_order();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 fb[NF];
#pragma unroll
            for (int j = 0; j < NF; ++j) fb[j] = read_b(lb, j, h);
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                const i32x4 a = h == 0 ? A::template read<0>(la, a_row(i), lane) : A::template read<1>(la, a_row(i), lane);
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[j]), __builtin_bit_cast(bf16x8, a),
                                                                        acc[i][j], 0, 0, 0);
            }
        }
        arrive<B::kLoads>();                               // the next step's rows; the weights' loads go on
        fetch_a(s + 2, d);
        in_order();
    };
    fetch_b(0, b[0]);
    fetch_b(1, b[1]);
    b[0].template store<0>(lds[0] + T::M * kStepBytes, tid);
    b[0].template store<1>(lds[0] + T::M * kStepBytes, tid);
    fetch_b(2, b[0]);
    in_order();
    fetch_a(0, 0);
    in_order();
    fetch_a(1, 1);
    in_order();
    arrive<A::kLoads>();
    for (int64_t s = 0; s < steps; s += 2) {               // past the last step: zeros
        step(s, Const<0>{});
        step(s + 1, Const<1>{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load into LDS outlives the workgroup

    const float S = p.S[t.expert];
    if (!p.out_f32 && p.outer % 8 == 0) {
        // through LDS, as whole rows of the tile
        constexpr int kOutChunks = T::N / 8, kMask = 15;
        static_assert(kRows * T::N * 2 <= kSteps * (T::M + T::N) * kStepBytes, "the tile in LDS");
        char* tile = lds[0];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const f32x4 v = acc[i][j] * S;
                const int row = a_row(i) + lane % 16, col = b_row(j) + lane / 16 * 4;
                *reinterpret_cast<uint2*>(tile + (row * kOutChunks + ((col / 8) ^ (row & kMask))) * kChunk + col % 8 * 2) =
                    make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
            }
        __syncthreads();
#pragma unroll 4
        for (int c = tid; c < kRows * kOutChunks; c += T::kThreads) {
            const int row = c / kOutChunks, chunk = c % kOutChunks;
            const int64_t n = n0 + chunk * 8;
            if (row < t.left && n < p.outer)
                *reinterpret_cast<i32x4*>(static_cast<uint16_t*>(p.out) + (t.first + row) * p.outer + n) =
                    *reinterpret_cast<const i32x4*>(tile + (row * kOutChunks + (chunk ^ (row & kMask))) * kChunk);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t row = a_row(i) + lane % 16;
        if (row >= t.left) continue;
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            const int64_t n = n0 + b_row(j) + lane / 16 * 4;
            store4(p.out, p.out_f32, (t.first + row) * p.outer + n, p.outer - n, p.outer % 4 == 0, acc[i][j] * S);
        }
    }
}

template <class T, bool TURNED, Scales SCALES>
__global__ __launch_bounds__(T::kThreads, 2) void grouped_kernel(Args p) {
    __shared__ __attribute__((aligned(1024))) char lds[kSteps][(T::M + T::N) * kStepBytes];
    const int tid = threadIdx.x;
    const Work work = work_of(blockIdx.x, gridDim.x, p.tiles_n);
    const int64_t n0 = work.n * T::N;
    const Place t = place_of(p, work.index, T::M, tid % kLanes);
    if (t.expert < 0) return clear_rows(p, t, n0, T::N, gridDim.x / p.tiles_n - (work.index - t.index), tid, T::kThreads);
    if constexpr (T::kLeast <= 1) if (t.left <= 32) return product<T, TURNED, SCALES, 1>(p, t, n0, lds, tid);
    if constexpr (T::kLeast <= 2) if (t.left <= 64) return product<T, TURNED, SCALES, 2>(p, t, n0, lds, tid);
    if constexpr (T::kMost > 4) if (t.left <= 128) return product<T, TURNED, SCALES, 4>(p, t, n0, lds, tid);
    product<T, TURNED, SCALES, T::kMost>(p, t, n0, lds, tid);
}

}  // namespace grouped_product
