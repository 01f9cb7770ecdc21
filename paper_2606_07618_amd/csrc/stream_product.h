// NVFP4 products with some to some hundreds of activation rows: the weights are read once for each 128 rows and
// expanded in registers, on their way into the matrix instructions, so no expanded copy of them is written.
//
// A weight q s has six significant bits and lies in 2^-10 .. 2688: exact in bfloat16, the activations' own type, which
// the matrix instructions take as they are.  (Binary16 would take half of the expansion's instructions, but it spans
// 40 powers of two: beside one large value of a row its small ones are lost.  It also needs a launch that scales the rows.
// [48, 4096] x [14336, 4096]: 23.6 us so, 21.9 in bfloat16; [16, 8192] x [28672, 8192]: 48 and 49.)
//
// A workgroup owns 128 weight rows and up to 128 activation rows.  Its waves are four times 32 weight rows by the
// two halves of its contraction; a wave loads its weights (32 rows by two lanes of 16 bytes) into
// registers, kAhead groups ahead, and all waves share a step's activations in LDS, D - 1 steps ahead; a step waits
// for what was started then and for nothing later.  The halves' sums meet in LDS at the end.
// Weights are loaded by groups of 256 values of a row, whole lines of 128 bytes, and so are the group's scales
// where their rows allow it: visited in smaller pieces, a line would have left the L1 between two visits.
// Few weight rows: the contraction is split over workgroups as well, whose sums a second kernel adds in order.
// [48, 8192] x [28672, 8192]: 59 us (2.3 TB/s, 0.38 PFLOP/s); 231 us with the weights expanded beforehand.  Neither
// the matrix instructions (20 % of the chip's cycles) nor the vector ones (32 %) bound it, nor do the bytes: with one
// group ahead and one workgroup on each of 224 compute units, too few weights are on their way.
#pragma once

#include "tile_product.h"

namespace stream_product {

using namespace tile_product;

using product_plan::kStreamRowsN, product_plan::kWavesK, product_plan::kGroup;
constexpr int kRowsN = kStreamRowsN;             // weight rows of a workgroup, 32 a wave
constexpr int kPiece = 64;                       // values of a weight row in one load of a wave

struct Args {
    const char* q;
    const uint8_t* scales;
    const char* x;                               // [m, ldx bytes]
    int64_t ldx, m, n, k;
    int64_t tiles_n;
    int parts, tiles_m, shift, part_values;      // part_values: of the contraction, a part
    const float* scale;
    void* out;
    int out_f32;
};

// Eight values times their scale, exact: the upper half of the binary32 product holds all of it.
__device__ __forceinline__ bf16x8 expand8(uint32_t n, float s) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, 1.0f, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(n, 1.0f, 3);
    const auto top = [&](f32x2 p) { return (int)__builtin_amdgcn_perm(__float_as_uint(p[1] * s), __float_as_uint(p[0] * s), 0x07060302u); };
    const i32x4 v = {top(a), top(b), top(c), top(d)};
    return __builtin_bit_cast(bf16x8, v);
}

// How a lane gets its scales: those of a whole group of its row (blocks of 16: four words, of 32: two), or of its
// own 32 values, one or two; kOdd: k is an odd multiple of 16, and a lane's 16 bytes may be half outside.
enum Scales { kWide16, kWide32, kPair, kOne, kOdd };

// MF: 32 activation rows each.
template <int MF, Scales SCALES>
__global__ __launch_bounds__(256 * kWavesK, kWavesK) void stream_kernel(Args p) {
    constexpr bool WIDE = SCALES == kWide16 || SCALES == kWide32, PAIRS = SCALES == kWide16 || SCALES == kPair || SCALES == kOdd;
    constexpr int A = MF == 4 ? 1 : 2;           // pieces of a wave in a step
    constexpr int D = 4, kTurn = MF == 4 ? 8 : 4;              // kTurn: steps after which slots and registers recur
    constexpr int kThreads = 256 * kWavesK, kStep = kPiece * A, kChunks = kStep * kWavesK / 8;   // chunks of a row
    constexpr int kStage = MF * 32 * kChunks * kChunk, kX = kStage / (kThreads * kChunk);
    constexpr int kPieces = kGroup / kPiece, G = kGroup / kStep;             // of a group; steps of a group
    constexpr int kGroups = kTurn / G, kAhead = 1;
    constexpr int kWords = SCALES == kWide16 ? 4 : SCALES == kWide32 ? 2 : kPieces;
    // loads of a group; kOdd's halves are left out of the count, which can only make a wait longer
    constexpr int kLoads = SCALES == kOdd ? 0 : kPieces + (WIDE ? 1 : kPieces);
    __shared__ __attribute__((aligned(1024))) char lds[D][kStage];
    static_assert((kWavesK - 1) * 4 * MF * 16 * kLanes * 4 <= D * kStage, "the other half's sums");

    const int tid = threadIdx.x, lane = tid % kLanes, g = lane / 32, i32 = lane % 32;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes), r = wave % 4, h = wave / 4;
    // neighbouring workgroups take the same weights for other activation rows
    const int64_t tile_m = blockIdx.x % p.tiles_m, rest = blockIdx.x / p.tiles_m;
    const int64_t n0 = rest % p.tiles_n * kRowsN, part = rest / p.tiles_n, m0 = tile_m * MF * 32;
    const int k = (int)p.k, half = p.part_values / kWavesK, begin = (int)part * p.part_values;
    const int k_begin = begin + h * half, k_end = k_begin + half < k ? k_begin + half : k;
    const int steps = ((half < k - begin ? half : k - begin) + kStep - 1) / kStep;   // the first half is the longer one

    const uint32_t q_ld = (uint32_t)k / 2, s_ld = (uint32_t)k >> p.shift;
    const __amdgpu_buffer_rsrc_t rq = window(p.q + n0 * q_ld), rs = window(p.scales + n0 * s_ld), rx = window(p.x + m0 * p.ldx);
    const int row = r * 32 + i32;
    // offsets of rows that are not there stay outside with any column added
    const uint32_t q_row = n0 + row < p.n ? (uint32_t)row * q_ld : kOutside, s_row = n0 + row < p.n ? (uint32_t)row * s_ld : kOutside;
    uint32_t x_row[kX];
    int x_left[kX];                              // values from the chunk's first place to its half's end
#pragma unroll
    for (int i = 0; i < kX; ++i) {
        // a chunk's place in its row is exchanged by the row: 16 lanes read one chunk of 16 rows
        const int id = i * kThreads + tid, xr = id / kChunks, chunk = id % kChunks ^ xr % 16;
        const int from = begin + chunk / (kStep / 8) * half, at = from + chunk % (kStep / 8) * 8;
        x_row[i] = m0 + xr < p.m ? (uint32_t)xr * (uint32_t)p.ldx + at * 2 : kOutside;
        x_left[i] = (from + half < k ? from + half : k) - at;
    }

    i32x4 w[kGroups][kPieces];
    uint32_t sc[kGroups][kWords];
    auto fetch_weights = [&](int group, auto to) {
        constexpr int T = decltype(to)::value;
        const int k0 = k_begin + group * kGroup;
#pragma unroll
        for (int a = 0; a < kPieces; ++a) {
            const int v = k0 + a * kPiece + g * 32;        // this lane's 32 values
            const bool in0 = v < k_end;
            const uint32_t q_at = q_row + (uint32_t)v / 2;
            if constexpr (SCALES == kOdd) {
                const i32x2 lo = load8(rq, in0 ? q_at : kOutside), hi = load8(rq, v + 16 < k_end ? q_at + 8 : kOutside);
                w[T][a] = i32x4{lo[0], lo[1], hi[0], hi[1]};
            } else {
                w[T][a] = load16(rq, in0 ? q_at : kOutside);
            }
            if constexpr (!WIDE) {
                const uint32_t s_at = s_row + ((uint32_t)v >> p.shift);
                if constexpr (SCALES == kOne) sc[T][a] = load1(rs, in0 ? s_at : kOutside);
                else if constexpr (SCALES == kPair)
                    sc[T][a] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(in0 ? s_at : kOutside), 0, 0);
                else sc[T][a] = load1(rs, in0 ? s_at : kOutside) | load1(rs, v + 16 < k_end ? s_at + 1 : kOutside) << 8;
            }
        }
        if constexpr (SCALES == kWide16) {                 // k is a multiple of the group
            const i32x4 c = load16(rs, k0 < k_end ? s_row + (uint32_t)k0 / 16 : kOutside);
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[T][j] = (uint32_t)c[j];
        }
        if constexpr (SCALES == kWide32) {
            const i32x2 c = load8(rs, k0 < k_end ? s_row + (uint32_t)k0 / 32 : kOutside);
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[T][j] = (uint32_t)c[j];
        }
    };
    auto fetch_x = [&](int s, int slot) {
#pragma unroll
        for (int i = 0; i < kX; ++i) {
            const uint32_t off = s * kStep < x_left[i] ? x_row[i] + (uint32_t)s * (kStep * 2) : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void*)(lds[slot] + (i * kThreads + wave * kLanes) * kChunk), kChunk,
                                                     (int)off, 0, 0, 0);
        }
    };
    // what step s (d of its turn) starts: a group's weights in a group's first step, then a later step's activations
    auto fetch = [&](int s, auto dc) {
        constexpr int d = decltype(dc)::value;
        if constexpr (d % G == 0) fetch_weights(s / G + kAhead, Const<(d / G + kAhead) % kGroups>{});
        fetch_x(s + D - 1, (d + D - 1) % D);
    };

    f32x16 acc[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;

    // Registers: the activations of four matrix instructions along the contraction, read two ahead of their use.
    bf16x8 xv[4][MF];
    int x_lane = (i32 * kChunks + ((h * A * 8 + g * 4) ^ i32 % 16)) * kChunk;      // of piece 0, instruction 0
    auto read = [&](int slot, int a, int j) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            xv[j][i] = *reinterpret_cast<const bf16x8*>(lds[slot] + i * (32 * kChunks * kChunk) + (x_lane ^ (a * 8 + j) * kChunk));
        }
    };
    // One step; past the last one it multiplies zeros.
    auto step = [&](int s, auto dc) {
        constexpr int d = decltype(dc)::value, slot = d % D;
        asm volatile("" : "+v"(x_lane));                   // addresses are made in each step, not kept for all
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int piece = d % G * A + a;               // of the group
            uint32_t c;                                    // blocks of 16: two codes, else one
            if constexpr (SCALES == kWide16) c = sc[d / G][piece] >> (g * 16);
            else if constexpr (SCALES == kWide32) c = sc[d / G][piece / 2] >> (piece % 2 * 16 + g * 8);
            else c = sc[d / G][piece];
            const float f0 = e4m3_f32(c), f1 = PAIRS ? e4m3_f32(c >> 8) : f0;
            if (a == A - 1) {
                // the next step's activations are here, the last one's are read; later loads: of the D - 3 steps before
                constexpr int first = d + 3 - D + kTurn, last = d - 1 + kTurn;   // of the turn before, on
                constexpr int kStarts = last / G - (first - 1) / G;          // groups begun in them
                arrive<(D - 3) * kX + kStarts * kLoads>();
                fetch(s, dc);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < 2) read(slot, a, j + 2);
                else read(a == A - 1 ? (d + 1) % D : slot, a == A - 1 ? 0 : a + 1, j - 2);
                int n = w[d / G][piece][j];
                // with many accumulators: expanded here, where its registers are needed, not a step ahead
                if constexpr (MF > 1) asm volatile("" : "+v"(n));
                bf16x8 wv = expand8((uint32_t)n, j < 2 ? f0 : f1);
                if constexpr (MF > 1) asm volatile("" : "+v"(wv));
#pragma unroll
                for (int i = 0; i < MF; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv, xv[j][i], acc[i], 0, 0, 0);
            }
        }
    };
    // What the steps before the first one would have started, in their order: the waits count on it.
    auto in_order = [] { asm volatile("" ::: "memory"); };
    static_assert(kAhead == 1 && kGroups == 2, "one group ahead");
#pragma unroll
    for (int d = 0; d < D - 1; ++d) {
        if (d == (G < D - 1 ? D - 1 - G : 0)) fetch_weights(0, Const<0>{});
        in_order();
        fetch_x(d, d);
        in_order();
    }
    arrive<(D - 2) * kX>();
#pragma unroll
    for (int j = 0; j < 2; ++j) read(0, 0, j);
    for (int s = 0; s < steps; s += kTurn) {
        step(s, Const<0>{}), step(s + 1, Const<1>{}), step(s + 2, Const<2>{}), step(s + 3, Const<3>{});
        if constexpr (kTurn == 8) step(s + 4, Const<4>{}), step(s + 5, Const<5>{}), step(s + 6, Const<6>{}), step(s + 7, Const<7>{});
    }

    arrive<0>();
    float* sums = reinterpret_cast<float*>(lds[0]);        // [kWavesK - 1][4][MF][16][lanes]
    if (h > 0) {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[((((h - 1) * 4 + r) * MF + i) * 16 + e) * kLanes + lane] = acc[i][e];
    }
    __syncthreads();
    if (h > 0) return;
#pragma unroll
    for (int o = 0; o < kWavesK - 1; ++o)
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][e] += sums[(((o * 4 + r) * MF + i) * 16 + e) * kLanes + lane];
    const float scale = *p.scale;
    const bool vec = p.n % 4 == 0;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t m = m0 + i * 32 + i32;
        if (m >= p.m) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = {acc[i][q * 4], acc[i][q * 4 + 1], acc[i][q * 4 + 2], acc[i][q * 4 + 3]};
            const int64_t n = n0 + r * 32 + q * 8 + g * 4;
            store4(p.out, p.parts > 1 || p.out_f32, ((p.parts > 1 ? part * p.m : 0) + m) * p.n + n, p.n - n, vec, v * scale);
        }
    }
}

}  // namespace stream_product
