// NVFP4 products with some tens or hundreds of activation rows: the weights are read once for each 128 rows and
// expanded in registers, on their way into the matrix instructions, so no expanded copy of them is written.
//
// A workgroup owns 128 weight rows and up to 128 activation rows.  Its waves are four times 32 weight rows by KW
// parts of each step of the contraction (64 values each); a wave loads its weights (32 rows by two lanes of
// 16 bytes) into registers, D steps ahead, and all waves share the step's activations in LDS, as many steps
// ahead, so that a step's wait is for what was started D - 1 steps before.  The parts' sums meet in LDS at the end.
// Few weight rows: the contraction is split over workgroups as well, whose sums a second kernel adds in order.
#pragma once

#include "thin_product.h"

namespace stream_product {

using namespace tile_product;
using thin_product::e4m3_f32;
using thin_product::expand8;
using thin_product::i32x2;
using thin_product::load1;
using thin_product::load16;
using thin_product::load8;

constexpr int kRowsN = 128;                      // weight rows of a workgroup, 32 a wave
constexpr int kWavesK = 2;                       // waves along a step

struct Args {
    const char* q;
    const uint8_t* scales;
    const char* x;                               // [m, ldx bytes]
    int64_t ldx, m, n, k;
    int64_t steps, split_steps, tiles_n;
    int parts, tiles_m, shift;
    const float* scale;
    void* out;
    int out_f32;
};

// MF: 32 activation rows each.  EVEN: k is a multiple of 32.  PAIRS: blocks of 16, two scales a lane.
template <int MF, bool EVEN, bool PAIRS>
__global__ __launch_bounds__(256 * kWavesK, kWavesK) void stream_kernel(Args p) {
    constexpr int KW = kWavesK, D = MF == 4 ? 5 : 8;
    constexpr int kThreads = 256 * KW, kStep = 64 * KW, kChunks = 8 * KW;      // of a row of a step
    constexpr int kStage = MF * 32 * kStep * 2;
    constexpr int kLeast = 2 + MF;               // loads of a step, at least
    __shared__ __attribute__((aligned(1024))) char lds[D][kStage];
    static_assert((KW - 1) * 4 * MF * 16 * kLanes * 4 <= D * kStage, "the other parts' sums");

    const int tid = threadIdx.x, lane = tid % kLanes, g = lane / 32, i32 = lane % 32;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes), r = wave % 4, h = wave / 4;
    // neighbouring workgroups take the same weights for other activation rows
    const int64_t tile_m = blockIdx.x % p.tiles_m, rest = blockIdx.x / p.tiles_m;
    const int64_t n0 = rest % p.tiles_n * kRowsN, part = rest / p.tiles_n, m0 = tile_m * MF * 32;
    const int64_t s0 = part * p.split_steps;
    const int64_t s1 = s0 + p.split_steps < p.steps ? s0 + p.split_steps : p.steps;

    const uint32_t q_ld = (uint32_t)(p.k / 2), s_ld = (uint32_t)(p.k >> p.shift);
    const __amdgpu_buffer_rsrc_t rq = window(p.q + n0 * q_ld), rs = window(p.scales + n0 * s_ld), rx = window(p.x + m0 * p.ldx);
    const int row = r * 32 + i32;
    const bool row_in = n0 + row < p.n;
    const uint32_t q_row = (uint32_t)row * q_ld, s_row = (uint32_t)row * s_ld;

    i32x4 w[D];
    uint32_t sc[D];
    auto fetch = [&](int64_t s, int slot) {
        const int64_t k0 = s * kStep;
        const int64_t v = k0 + h * 64 + g * 32;                // this lane's 32 values
        const bool in0 = row_in && s < s1 && v < p.k, in1 = EVEN ? in0 : in0 && v + 16 < p.k;
        if constexpr (EVEN) {
            w[slot] = load16(rq, in0 ? q_row + (uint32_t)v / 2 : kOutside);
        } else {
            const i32x2 lo = load8(rq, in0 ? q_row + (uint32_t)v / 2 : kOutside), hi = load8(rq, in1 ? q_row + (uint32_t)v / 2 + 8 : kOutside);
            w[slot] = i32x4{lo[0], lo[1], hi[0], hi[1]};
        }
        if constexpr (!PAIRS) sc[slot] = load1(rs, in0 ? s_row + (uint32_t)(v >> p.shift) : kOutside);
        else if constexpr (EVEN)
            sc[slot] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, (int)(in0 ? s_row + (uint32_t)(v >> 4) : kOutside), 0, 0);
        else sc[slot] = load1(rs, in0 ? s_row + (uint32_t)(v >> 4) : kOutside) |
                        load1(rs, in1 ? s_row + (uint32_t)(v >> 4) + 1 : kOutside) << 8;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            // a chunk's place in its row is exchanged by the row: 16 lanes read one chunk of 16 rows
            const int id = i * kThreads + tid, xr = id / kChunks, chunk = id % kChunks ^ xr % 16;
            const bool in = m0 + xr < p.m && s < s1 && k0 + chunk * 8 < p.k;
            const uint32_t off = in ? (uint32_t)xr * (uint32_t)p.ldx + (uint32_t)(k0 + chunk * 8) * 2 : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void*)(lds[slot] + (i * kThreads + wave * kLanes) * kChunk), kChunk,
                                                     (int)off, 0, 0, 0);
        }
    };

    f32x16 acc[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;

    // Registers: this step's activations and the next one's, read while this one's are multiplied.
    bf16x8 xv[2][4][MF];
    auto read = [&](int slot, int to, int j) {
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int chunk = (h * 8 + g * 4 + j) ^ i32 % 16;
            xv[to][j][i] = *reinterpret_cast<const bf16x8*>(lds[slot] + (i * 32 + i32) * (kStep * 2) + chunk * kChunk);
        }
    };
#pragma unroll
    for (int d = 0; d < D - 1; ++d) fetch(s0 + d, d);
    arrive<(D - 2) * kLeast>();
#pragma unroll
    for (int j = 0; j < 4; ++j) read(0, 0, j);
    constexpr int kTurn = D % 2 ? 2 * D : D;     // steps after which slots and registers recur
    for (int64_t s = s0; s < s1; s += kTurn) {
#pragma unroll
        for (int d = 0; d < kTurn; ++d) {
            if (s + d >= s1) break;
            arrive<(D - 3) * kLeast>();          // the next step's activations are here, this one's are read
            fetch(s + d + D - 1, (d + D - 1) % D);
            const int slot = d % D;
            const float f0 = e4m3_f32(sc[slot]), f1 = PAIRS ? e4m3_f32(sc[slot] >> 8) : f0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                read((d + 1) % D, (d + 1) % 2, j);
                const bf16x8 wv = expand8((uint32_t)w[slot][j], j < 2 ? f0 : f1);
#pragma unroll
                for (int i = 0; i < MF; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv, xv[d % 2][j][i], acc[i], 0, 0, 0);
            }
        }
    }

    arrive<0>();
    float* sums = reinterpret_cast<float*>(lds[0]);      // [KW - 1][4][MF][16][lanes]
    if (h > 0) {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[((((h - 1) * 4 + r) * MF + i) * 16 + e) * kLanes + lane] = acc[i][e];
    }
    __syncthreads();
    if (h > 0) return;
#pragma unroll
    for (int o = 0; o < KW - 1; ++o)
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][e] += sums[(((o * 4 + r) * MF + i) * 16 + e) * kLanes + lane];
    const float scale = p.parts == 1 && p.scale ? *p.scale : 1.0f;
    const bool vec = p.n % 4 == 0;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t m = m0 + i * 32 + i32;
        if (m >= p.m) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = f32x4{acc[i][q * 4], acc[i][q * 4 + 1], acc[i][q * 4 + 2], acc[i][q * 4 + 3]} * scale;
            const int64_t n = n0 + r * 32 + q * 8 + g * 4;
            store4(p.out, p.parts > 1 || p.out_f32, ((p.parts > 1 ? part * p.m : 0) + m) * p.n + n, p.n - n, vec, v);
        }
    }
}

inline int rows_of(int64_t m) { return m <= 32 ? 1 : m <= 64 ? 2 : 4; }
inline int tiles_m(int64_t m) { return (int)((m + 127) / 128); }
inline int64_t steps(int64_t k) { return (k + 64 * kWavesK - 1) / (64 * kWavesK); }
// A workgroup takes a compute unit's LDS: parts of the contraction, of at least eight steps, until 256 units
// have work.
inline int parts(int64_t m, int64_t n, int64_t k) {
    const int64_t groups = (n + kRowsN - 1) / kRowsN * tiles_m(m);
    int64_t want = (256 + groups / 2) / (groups ? groups : 1);
    if (want > steps(k) / 8) want = steps(k) / 8;
    if (want > 16) want = 16;
    return want < 1 ? 1 : (int)want;
}

}  // namespace stream_product
