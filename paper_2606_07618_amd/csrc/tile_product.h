// Tiled matrix product on the matrix cores of gfx950, D[m][n] = sum_k A[m][k] B[n][k], sums in
// binary32, for bfloat16 operands and for microscaled FP4 ones (E2M1 nibbles with an E8M0 scale
// for each 32 values of a row); and for 8-bit integers, sums in 32-bit integers.  Both operands' rows hold the contraction; what is done with the sums is a
// template argument.  (A contraction that runs down an operand's rows is turned before: with the matrix
// turned inside the product, by transposing reads of LDS, a step took 1.5 us in place of 1.0, and a
// gradient of [4096, 14336] x [14336, 4096] 438 us in place of 360, of which 37 for the turning.)
//
// All element types share one geometry: a step takes 128 bytes of every row of the tile (64
// bfloat16 values, 128 integers, 256 FP4 ones), and a lane's operand of one matrix instruction is 16 of them (8
// values of 16x16x32, 16 of 16x16x64, 32 of 16x16x128), so staging, LDS layout and register tiles are the same.
// (On random values the card's power holds 16x16 instructions at 2.13 PFLOP/s bfloat16 and 7.5 FP4, the
// 32x32 ones at 1.86 and 6.3.)
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "product_plan.h"

namespace tile_product {

using product_plan::Kind, product_plan::kBf16, product_plan::kMx, product_plan::kMxLaid, product_plan::kInt8;
using product_plan::Out, product_plan::kSums, product_plan::kPartial, product_plan::kGate, product_plan::kGatePartial,
    product_plan::kTwoRows, product_plan::kAdded;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

typedef __attribute__((address_space(3))) void lds_void;

constexpr int kLanes = 64;
constexpr int kStepBytes = 128;                  // of a row, a step of the contraction
constexpr int kChunk = 16;                       // bytes of a lane's load
constexpr uint32_t kOutside = 0x80000000u;       // an offset that the buffer's size excludes: reads as zero

// A window of 2 GiB from `base`: loads at offsets of kOutside and up return zero without an access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)kOutside, 0x00020000);
}

// Loads at such offsets into registers.
__device__ __forceinline__ i32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)at, 0, 0));
}
__device__ __forceinline__ i32x2 load8(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return __builtin_bit_cast(i32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)at, 0, 0));
}
__device__ __forceinline__ uint32_t load1(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(r, (int)at, 0, 0);
}

// An E4M3 number times 2^UP.
template <int UP = 0>
__device__ __forceinline__ float e4m3_f32(uint32_t c) {
    // the code's fields as those of a binary32 number 2^120 times too small; the product is exact
    return __uint_as_float((c & 0x7Fu) << 20) * __builtin_ldexpf(0x1p120f, UP);
}

template <int V> struct Const { static constexpr int value = V; };

struct Operand {
    const char* p;              // element (0, 0)
    const char* p2;             // the second matrix (B of kGate)
    int64_t ld;                 // bytes from row to row
    const uint8_t* scales;      // microscaled: E8M0 codes
    int64_t scale_ld;           // kMx: bytes from row to row
};

__device__ __forceinline__ float silu(float g) {
    // g / (1 + e^-g): e^-g overflows to infinity below -88, where the quotient's reciprocal is zero.
    const float e = __builtin_amdgcn_exp2f(g * -1.44269504f);
    return g * __builtin_amdgcn_rcpf(1.0f + e);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// E8M0 codes in the order in which lanes take them: for the 16 F rows of a wave's fragments and for a step, each lane's
// codes of its F fragments, two neighbouring bytes a fragment (blocks lane / 16 and 4 + lane / 16 of the step), so that
// an instruction picks its byte from a word as it was read.  As the rows lie, a step takes eight bytes of each row's
// scales, whose lines, fetched again for each step, are as many bytes as the values themselves: with a chip full of
// the largest tiles this costs more than laying the scales out ([8192, 4096] x [14336, 4096]: 313 us as they lie,
// 271 laid out, 7 of them for that; [64, 4096] x [14336, 4096]: 14.5 and 16).
__device__ __forceinline__ int64_t scale_at(int64_t group, int64_t steps, int64_t step, int lane, int fragments) {
    return ((group * steps + step) * kLanes + lane) * fragments * 2;
}

// All but this wave's last LEFT loads into LDS have arrived and its reads of LDS are done, then all waves'.
template <int LEFT>
__device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// The sequence of tiles: workgroups go to the eight XCDs in turn, so each XCD gets a contiguous run of
// the sequence, and the sequence walks kGroup tile rows at a time: what an XCD works on at one time shares
// rows of A and of B in its L2.
constexpr int kXcds = 8, kGroup = 8;
struct TileIndex { int64_t m, n; };
__device__ __forceinline__ TileIndex tile_of(int64_t id, int64_t count, int64_t tiles_m, int64_t tiles_n) {
    const int64_t xcd = id % kXcds, each = count / kXcds, rest = count % kXcds;
    const int64_t seq = xcd * each + (xcd < rest ? xcd : rest) + id / kXcds;
    const int64_t per_group = kGroup * tiles_n;
    const int64_t first = seq / per_group * kGroup;
    const int64_t height = tiles_m - first < kGroup ? tiles_m - first : kGroup;
    const int64_t in = seq % per_group;
    return {first + in % height, in / height};
}

// One operand's side of a tile: R outer indexes, staged by THREADS threads.
template <int R, int THREADS, bool HALF>
struct Side {
    static constexpr int kBytes = R * kStepBytes;
    static constexpr int kLoads = kBytes / (THREADS * kChunk);
    static_assert(kBytes % (THREADS * kChunk) == 0, "whole loads");
    static constexpr int kRowChunks = kStepBytes / kChunk;

    // LDS holds a step as rows of chunks.  A chunk's place in its row is exchanged by the row, so that
    // the lanes of a read hit all banks: 16 lanes read one chunk of 16 rows, and the row's parity and the
    // exchanged place cover the 256 bytes of the banks.
    __device__ static __forceinline__ int exchange(int row) { return (row >> 1) & 7; }

    uint32_t offset[kLoads];             // of this thread's loads from the step's base

    // left: the outer indexes from the tile's first one on.  With HALF, rows from R / 2 on are the same
    // outer indexes of the second matrix.
    __device__ __forceinline__ void init(int64_t left, int64_t ld, int tid) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = i * THREADS + tid, row = id / kRowChunks;
            const int chunk = (id % kRowChunks) ^ exchange(row);
            const int r = HALF ? row % (R / 2) : row;
            offset[i] = r < left ? (uint32_t)r * (uint32_t)ld + chunk * kChunk : kOutside;
        }
    }

    // Starts the loads of one step into LDS.  ahead: bytes of a row from the step's first one on; beyond
    // them LDS gets zeros.
    __device__ __forceinline__ void load(const char* base, const char* base2, char* lds, int64_t ahead, int tid,
                                         int wave) const {
        const __amdgpu_buffer_rsrc_t w = window(base), w2 = HALF ? window(base2) : w;
        const int left = ahead > kStepBytes ? kStepBytes : ahead > 0 ? (int)ahead : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool second = HALF && i * THREADS / kRowChunks >= R / 2;
            const int id = i * THREADS + tid, row = id / kRowChunks;
            const int at = ((id % kRowChunks) ^ exchange(row)) * kChunk;
            const uint32_t off = at < left ? offset[i] : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? w2 : w,
                                                     (lds_void*)(lds + (i * THREADS + wave * kLanes) * kChunk), kChunk,
                                                     (int)off, 0, 0, 0);
        }
    }

    // This lane's 16 bytes of the operand at outer indexes row0 .. row0 + 15 of the tile, half H of the step.
    // bfloat16: values 32 H + 8 (lane / 16) on.  Microscaled: the 32-value block 4 H + lane / 16.
    template <int H>
    __device__ static __forceinline__ i32x4 read(const char* lds, int row0, int lane) {
        const int row = row0 + lane % 16, chunk = 4 * H + lane / 16;
        return *reinterpret_cast<const i32x4*>(lds + row * kStepBytes + ((chunk ^ exchange(row)) * kChunk));
    }
};

// Workgroup tile M_ x N_ by WM x WN waves.
template <int M_, int N_, int WM_, int WN_, int SLOTS = 2>
struct Tile {
    static constexpr int kSlots = SLOTS;                             // steps of the contraction in LDS
    static constexpr int M = M_, N = N_, WM = WM_, WN = WN_, kThreads = WM_ * WN_ * kLanes;
    static constexpr int kWavesPerSimd = M_ * N_ / (WM_ * WN_) > 8192 ? 1 : 2;   // 512 or 256 registers
    static constexpr int MF = M_ / WM_ / 16, NF = N_ / WN_ / 16;     // a wave's matrix instructions
};

struct Args {
    Operand a, b;
    int64_t m, n;               // outer indexes of A and of B (kGate: of each of B's two)
    int64_t inner;              // values of the contraction
    int64_t steps, split_steps; // of the whole contraction, and of one part of it
    int64_t tiles_m, tiles_n;
    int parts;
    int out_f32;
    const float* scale;         // NULL: 1
    const float *scale_m, *scale_n;      // kInt8: of the outer indexes of A and of B
    void *out, *out2, *out3;
    int64_t half_rows;          // kTwoRows
    int64_t out_ld;
};

__device__ __forceinline__ void store4(void* out, int f32, int64_t at, int64_t left, bool vec, f32x4 v) {
    if (f32) {
        float* o = static_cast<float*>(out) + at;
        if (vec && left >= 4) { *reinterpret_cast<f32x4*>(o) = v; return; }
#pragma unroll
        for (int r = 0; r < 4; ++r) if (r < left) o[r] = v[r];
    } else {
        const uint2 p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        uint16_t* o = static_cast<uint16_t*>(out) + at;
        if (vec && left >= 4) { *reinterpret_cast<uint2*>(o) = p; return; }
        if (left > 0) o[0] = (uint16_t)p.x;
        if (left > 1) o[1] = (uint16_t)(p.x >> 16);
        if (left > 2) o[2] = (uint16_t)p.y;
        if (left > 3) o[3] = (uint16_t)(p.y >> 16);
    }
}

// A lane's sums of a matrix instruction.  Integers leave as the nearest binary32 numbers times the two scales, or, as
// parts, in the bits of a binary32 number.
template <Kind KIND> struct SumsOf { typedef f32x4 type; };
template <> struct SumsOf<kInt8> { typedef i32x4 type; };

// sum a b where the product of the scales a and b may lie outside binary32 and the output does not: the scales as numbers of 1/2
// to 1, whose powers of two come last.  The same bits as sum * (a * b) where it lies inside.
__device__ __forceinline__ float scaled(int sum, float a, float b) {
    const float parts = __builtin_amdgcn_frexp_mantf(a) * __builtin_amdgcn_frexp_mantf(b);
    return __builtin_ldexpf((float)sum * parts, __builtin_amdgcn_frexp_expf(a) + __builtin_amdgcn_frexp_expf(b));
}
// Whether the product of two such scales lies inside.
__device__ __forceinline__ bool moderate(float s) { return (uint32_t)(__builtin_amdgcn_frexp_expf(s) + 62) <= 124; }

// The scales of n .. n + 3, those that there are.
__device__ __forceinline__ f32x4 scales4(const float* s, int64_t n, int64_t left) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 4; ++r) if (r < left) v[r] = s[n + r];
    return v;
}

template <Kind KIND, Out OUT, class T>
__global__ __launch_bounds__(T::kThreads, T::kWavesPerSimd) void product_kernel(Args p) {
    constexpr bool HALF = OUT == kGate || OUT == kGatePartial;
    using A = Side<T::M, T::kThreads, false>;
    using B = Side<T::N, T::kThreads, HALF>;
    constexpr bool kScaled = product_plan::kMicroscaled<KIND>, kLaid = KIND == kMxLaid;
    constexpr int kScales = kScaled ? (T::M + T::N) * 8 : 0;           // eight bytes a row and step
    constexpr int kScaleLoads = (kScales + T::kThreads * 4 - 1) / (T::kThreads * 4);
    constexpr bool kEven = kScales % (T::kThreads * 4) == 0;               // else the last waves' last load is not one
    constexpr int kStage = A::kBytes + B::kBytes + kScales;
    constexpr int kSlots = T::kSlots;
    constexpr int kLoads = A::kLoads + B::kLoads + kScales / (T::kThreads * 4);   // of a step, every wave's
    __shared__ __attribute__((aligned(1024))) char lds[kSlots][kStage];
    constexpr int kOutN = HALF ? T::N / 2 : T::N;          // output columns of a tile
    constexpr int NF = T::NF, MF = T::MF;

    const int tid = threadIdx.x, lane = tid % kLanes;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int wm = wave / T::WN, wn = wave % T::WN;
    const int64_t tiles = p.tiles_m * p.tiles_n;
    const int64_t part = blockIdx.x / tiles;
    const TileIndex t = tile_of(blockIdx.x % tiles, tiles, p.tiles_m, p.tiles_n);
    const int64_t m0 = t.m * T::M, n0 = t.n * kOutN;
    const int64_t s0 = part * p.split_steps;
    const int64_t s1 = s0 + p.split_steps < p.steps ? s0 + p.split_steps : p.steps;

    A sa;
    B sb;
    sa.init(p.m - m0, p.a.ld, tid);
    sb.init(p.n - n0, p.b.ld, tid);
    // Scales: LDS holds a step's wave by wave, A's then B's.  Laid out, as they lie in memory; else a word holds a half's
    // four codes of a row, by row in the fragment, half, fragment, so that a lane reads its fragments' words at once.
    uint32_t scale_offset[kScaleLoads + 1];
    int scale_left[kScaleLoads + 1];               // kMx: bytes of the step ahead of the word
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        int word = i * T::kThreads + tid;
        const bool of_a = word < T::M * 2;
        word -= of_a ? 0 : T::M * 2;
        const int fragments = of_a ? MF : NF, group = word / (32 * fragments), in = word % (32 * fragments);
        const int64_t left = of_a ? p.m - m0 : p.n - n0;
        if constexpr (kLaid) {
            scale_offset[i] = group * 16 * fragments < left ? (uint32_t)scale_at(group, p.steps, 0, 0, fragments) + in * 4 : kOutside;
            scale_left[i] = 0;
        } else {
            const int row = (group * fragments + in % fragments) * 16 + in / (2 * fragments);
            scale_left[i] = in / fragments % 2 * 4;
            scale_offset[i] = row < left ? (uint32_t)row * (uint32_t)(of_a ? p.a.scale_ld : p.b.scale_ld) + scale_left[i] : kOutside;
        }
    }
    const char* a0 = p.a.p + m0 * p.a.ld;
    const int64_t b_at = n0 * p.b.ld, row_bytes = kScaled ? p.inner / 2 : KIND == kInt8 ? p.inner : p.inner * 2;
    auto fetch_a = [&](int64_t s, int stage) {
        sa.load(a0 + s * kStepBytes, nullptr, lds[stage], row_bytes - s * kStepBytes, tid, wave);
    };
    auto fetch_b = [&](int64_t s, int stage) {
        char* l = lds[stage] + A::kBytes;
        const int64_t at = b_at + s * kStepBytes;
        sb.load(p.b.p + at, HALF ? p.b.p2 + at : nullptr, l, row_bytes - s * kStepBytes, tid, wave);
        if constexpr (kScaled) {
            const int64_t left = p.inner / 32 - s * 8;
            const __amdgpu_buffer_rsrc_t
                ra = window(p.a.scales + (kLaid ? scale_at(m0 / (16 * MF), p.steps, s, 0, MF) : m0 * p.a.scale_ld + s * 8)),
                rb = window(p.b.scales + (kLaid ? scale_at(n0 / (16 * NF), p.steps, s, 0, NF) : n0 * p.b.scale_ld + s * 8));
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i) {
                const int first = i * T::kThreads + wave * kLanes;
                if (!kEven && first * 4 >= kScales) break;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(first / 2 < T::M ? ra : rb, (lds_void*)(l + B::kBytes + first * 4), 4,
                                                         (int)(scale_left[i] < left ? scale_offset[i] : kOutside), 0, 0, 0);
            }
        }
    };

    // first rows of this wave's fragments in the tile
    auto a_row = [&](int i) { return wm * (T::M / T::WM) + i * 16; };
    auto b_row = [&](int j) {
        if constexpr (!HALF) return wn * (T::N / T::WN) + j * 16;
        return (j < NF / 2 ? 0 : T::N / 2) + wn * (T::N / 2 / T::WN) + j % (NF / 2) * 16;
    };

    using Sums = typename SumsOf<KIND>::type;
    Sums acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = Sums{0, 0, 0, 0};

    // A step is 2 MF groups of NF matrix instructions, a fragment of A against a half's fragments of B.
    // Registers run kLead groups ahead of them (a whole half for B), LDS kSlots steps: while a group is
    // multiplied a later one's fragment is read, and the one barrier of a step stands where its last fragments
    // have been read, so that its LDS is free for the step kSlots on.  That step's loads are started in two
    // parts, A's behind the barrier and B's in the next step, among the matrix instructions: in one burst
    // they fill the queue that both waves of a SIMD then wait at.  What a step waits for at its barrier are the
    // loads of the next step, and no later ones.
    constexpr int kLead = MF >= 8 ? 3 : MF >= 4 ? 2 : 1;
    constexpr int kRing = 4, kGroups = 2 * MF;
    i32x4 fa[kRing], fb[2][NF];
    // Codes of this step and the next step's words.  Laid out, a word is two fragments' codes of both halves; else a
    // half's of one fragment, and a lane picks its own.
    constexpr int kPer = kLaid ? 2 : 1, kHalves = kLaid ? 1 : 2;
    int xa[MF / kPer], xb[NF / kPer], ya[kHalves][MF / kPer], yb[kHalves][NF / kPer];
    auto read_a = [&](auto gc, int stage) {    // the fragment of group g of a step
        constexpr int g = decltype(gc)::value;
        fa[g % kRing] = A::template read<g / MF>(lds[stage], a_row(g % MF), lane);
    };
    auto read_b = [&](auto hc, int stage, int from, int to) {
        constexpr int H = decltype(hc)::value;
#pragma unroll
        for (int j = from; j < to; ++j) fb[H][j] = B::template read<H>(lds[stage] + A::kBytes, b_row(j), lane);
    };
    auto read_scales = [&](int stage) {
        if constexpr (kScaled) {
            const int* la = reinterpret_cast<const int*>(lds[stage] + A::kBytes + B::kBytes);
            const int at = kLaid ? lane : lane % 16 * 2, per = kLaid ? kLanes : 32;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
#pragma unroll
                for (int i = 0; i < MF / kPer; ++i) ya[h][i] = la[(wm * per + at + h) * (MF / kPer) + i];
#pragma unroll
                for (int j = 0; j < NF / kPer; ++j) yb[h][j] = la[T::M * 2 + (wn * per + at + h) * (NF / kPer) + j];
            }
        }
    };
    auto next_scales = [&]() {
        if constexpr (kScaled) {
            const uint32_t pick = 0x0C0C0400u + (uint32_t)(lane / 16) * 0x0101u;   // this lane's code of either half
            auto codes = [&](int first, int second) { return kLaid ? first : (int)__builtin_amdgcn_perm((uint32_t)second, (uint32_t)first, pick); };
#pragma unroll
            for (int i = 0; i < MF / kPer; ++i) xa[i] = codes(ya[0][i], ya[kHalves - 1][i]);
#pragma unroll
            for (int j = 0; j < NF / kPer; ++j) xb[j] = codes(yb[0][j], yb[kHalves - 1][j]);
        }
    };
    auto group = [&](int64_t s, int slot, int next, auto gc) {
        constexpr int g = decltype(gc)::value, H = g / MF, i = g % MF, ahead = g + kLead;
        constexpr bool first = ahead == kGroups;       // the first group whose reads ahead are the next step's
        // the second half's fragments of B: one in each of the first groups, or what is left in the last that may
        constexpr bool more_b = g < NF && g < MF - 1;
        constexpr int b_to = g == MF - 2 ? NF : g + 1;
        constexpr int kReads = 1 + (more_b ? b_to - g : 0) + (first ? NF + (kLaid ? 2 : kScaled ? (MF + NF) / 2 : 0) : 0);
        constexpr int kStarts = first ? A::kLoads : g == 0 ? B::kLoads : 0;
        if constexpr (first) {
            arrive<(kSlots - 2) * kLoads>();
            fetch_a(s + kSlots, slot);
            read_scales(next);
            read_b(Const<0>{}, next, 0, NF);
        }
        read_a(Const<ahead % kGroups>{}, ahead < kGroups ? slot : next);
        if constexpr (more_b) read_b(Const<1>{}, slot, g, b_to);
        if constexpr (g == 0) if (s > s0) fetch_b(s - 1 + kSlots, slot == 0 ? kSlots - 1 : slot - 1);
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            // B's values as the instruction's rows: a lane gets four neighbouring outputs of a row of D
            const i32x4 b = fb[H][j], a = fa[g % kRing];
            if constexpr (KIND == kInt8) {
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, acc[i][j], 0, 0, 0);
            } else if constexpr (!kScaled) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a),
                                                                    acc[i][j], 0, 0, 0);
            } else {
                const i32x8 wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0}, wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
                constexpr int kOdd = kLaid ? 2 : 0, kCode = i % 2 * kOdd + H;
                acc[i][j] = j % 2 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc[i][j], 4, 4, kOdd + H, xb[j / kPer], kCode, xa[i / kPer])
                                  : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc[i][j], 4, 4, H, xb[j / kPer], kCode, xa[i / kPer]);
            }
        }
        // the order of a group: its LDS reads and its loads among its matrix instructions
#pragma unroll
        for (int r = 0; r < NF; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, (kReads + NF - 1) / NF, 0);                          // LDS reads
            if constexpr (kStarts > 0) __builtin_amdgcn_sched_group_barrier(0x010, (kStarts + NF - 1) / NF, 0);  // loads from memory
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                               // matrix instructions
        }
    };
    if (s0 < s1) {
#pragma unroll
        for (int i = 0; i < kSlots; ++i) {
            fetch_a(s0 + i, i);                                      // past the contraction's end: zeros
            fetch_b(s0 + i, i);
            asm volatile("" ::: "memory");                           // the wait counts on this order
        }
        arrive<(kSlots - 1) * kLoads>();
        read_b(Const<0>{}, 0, 0, NF);
        read_scales(0);
        read_a(Const<0>{}, 0);
        if constexpr (kLead > 1) read_a(Const<1>{}, 0);
        if constexpr (kLead > 2) read_a(Const<2>{}, 0);
        int slot = 0;
        for (int64_t s = s0; s < s1; ++s) {
            const int next = slot + 1 == kSlots ? 0 : slot + 1;
            next_scales();
            group(s, slot, next, Const<0>{}), group(s, slot, next, Const<1>{});
            group(s, slot, next, Const<2>{}), group(s, slot, next, Const<3>{});
            if constexpr (MF >= 4) {
                group(s, slot, next, Const<4>{}), group(s, slot, next, Const<5>{});
                group(s, slot, next, Const<6>{}), group(s, slot, next, Const<7>{});
            }
            if constexpr (MF >= 8) {
                group(s, slot, next, Const<8>{}), group(s, slot, next, Const<9>{});
                group(s, slot, next, Const<10>{}), group(s, slot, next, Const<11>{});
                group(s, slot, next, Const<12>{}), group(s, slot, next, Const<13>{});
                group(s, slot, next, Const<14>{}), group(s, slot, next, Const<15>{});
            }
            static_assert(MF == 2 || MF == 4 || MF == 8, "groups of a step");
            slot = next;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // no load into LDS outlives the workgroup
    }

    // A lane holds four neighbouring columns of row lane % 16 of D.  Stored from here, an instruction would write
    // 32 bytes of 16 rows; bfloat16 outputs go through LDS instead and leave as whole rows of the tile, 16 bytes a
    // lane ([8192, 4096] x [14336, 4096] microscaled, where the contraction is short: 338 -> 305 us).  The largest tile,
    // whose outputs are too many to stay in the L2 until they are read, stores them past it and leaves the L2 to the
    // operands (the same product: 282 -> 252 us).
    const float scale = OUT == kSums && p.scale ? *p.scale : 1.0f;
    // integers: the scales of this lane's columns and of its rows.  A wave whose scales are all moderate multiplies them first
    // ([8192, 4096] x [14336, 4096] with its quantization: 396 us, 406 with powers of two for all).
    f32x4 scale_n[KIND == kInt8 && OUT == kSums ? NF : 1];
    float scale_m[KIND == kInt8 && OUT == kSums ? MF : 1];
    bool inside = true;
    if constexpr (KIND == kInt8 && OUT == kSums) {
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            const int64_t n = n0 + b_row(j) + lane / 16 * 4;
            scale_n[j] = scales4(p.scale_n, n, p.n - n);
#pragma unroll
            for (int e = 0; e < 4; ++e) inside = inside && moderate(scale_n[j][e]);
        }
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int64_t m = m0 + a_row(i) + lane % 16;
            scale_m[i] = m < p.m ? p.scale_m[m] : 0.0f;
            inside = inside && moderate(scale_m[i]);
        }
        inside = __all(inside);
    }
    auto sums = [&](int i, int j) {
        if constexpr (KIND != kInt8) return acc[i][j] * scale;
        else if constexpr (OUT != kSums) return __builtin_bit_cast(f32x4, acc[i][j]);
        else {
            const f32x4 s = scale_n[j] * scale_m[i];
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (float)acc[i][j][e] * s[e];
            return v;
        }
    };
    auto far_sums = [&](int i, int j) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (KIND == kInt8 && OUT == kSums) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = scaled(acc[i][j][e], scale_n[j][e], scale_m[i]);
        }
        return v;
    };
    auto column = [&](int j) { return HALF ? wn * (kOutN / T::WN) + j * 16 : b_row(j); };
    if (OUT != kPartial && OUT != kGatePartial && OUT != kAdded && !p.out_f32 && p.out_ld % 8 == 0) {
        constexpr int kOutChunks = kOutN / 8, kMask = kOutChunks < 16 ? kOutChunks - 1 : 15;
        static_assert(T::M * kOutN * 2 <= kSlots * kStage, "the tile in LDS");
        char* tile = lds[0];
        auto fill = [&](auto value) {
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < (HALF ? NF / 2 : NF); ++j) {
                    const f32x4 v = value(i, j);
                    const int row = a_row(i) + lane % 16, col = column(j) + lane / 16 * 4;
                    *reinterpret_cast<uint2*>(tile + (row * kOutChunks + ((col / 8) ^ (row & kMask))) * kChunk + col % 8 * 2) =
                        make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                }
        };
        auto write = [&](auto value, auto row_of) {      // value(i, j): of a fragment; row_of(m): where row m goes
            __syncthreads();
            if (inside) fill(value);                     // each wave by its own scales
            else fill(far_sums);
            __syncthreads();
#pragma unroll 4
            for (int c = tid; c < T::M * kOutChunks; c += T::kThreads) {
                const int row = c / kOutChunks, chunk = c % kOutChunks;
                const int64_t m = m0 + row, n = n0 + chunk * 8;
                if (m < p.m && n < p.n) {
                    const i32x4 v = *reinterpret_cast<const i32x4*>(tile + (row * kOutChunks + (chunk ^ (row & kMask))) * kChunk);
                    i32x4* to = reinterpret_cast<i32x4*>(row_of(m) + n);
                    if constexpr (T::M == 256) __builtin_nontemporal_store(v, to);
                    else *to = v;
                }
            }
        };
        auto rows_of = [&](void* out) { return [=](int64_t m) { return static_cast<uint16_t*>(out) + m * p.out_ld; }; };
        if constexpr (OUT == kSums) {
            write(sums, rows_of(p.out));
        } else if constexpr (OUT == kTwoRows) {
            write([&](int i, int j) { return acc[i][j]; }, [&](int64_t m) {
                return m < p.half_rows ? static_cast<uint16_t*>(p.out) + m * p.out_ld
                                       : static_cast<uint16_t*>(p.out2) + (m - p.half_rows) * p.out_ld;
            });
        } else if constexpr (OUT == kGate) {
            constexpr int H = NF / 2;
            write([&](int i, int j) {
                f32x4 h;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = silu(acc[i][j][e]) * acc[i][H + j][e];
                return h;
            }, rows_of(p.out));
            if (p.out2) {
                write([&](int i, int j) { return acc[i][j]; }, rows_of(p.out2));
                write([&](int i, int j) { return acc[i][H + j]; }, rows_of(p.out3));
            }
        }
        return;
    }
    const bool vec = p.out_ld % 4 == 0;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t m = m0 + a_row(i) + lane % 16;
        if (m >= p.m) continue;
#pragma unroll
        for (int j = 0; j < (HALF ? NF / 2 : NF); ++j) {
            const int64_t n = n0 + column(j) + lane / 16 * 4, left = p.n - n;
            f32x4 v;
            if constexpr (KIND == kInt8) v = inside ? sums(i, j) : far_sums(i, j);
            else v = acc[i][j];
            if constexpr (OUT == kSums) {
                store4(p.out, p.out_f32, m * p.out_ld + n, left, vec, KIND == kInt8 ? v : v * scale);
            } else if constexpr (OUT == kAdded) {
                const float* held = static_cast<const float*>(p.out) + m * p.out_ld + n;
#pragma unroll
                for (int e = 0; e < 4; ++e) if (e < left) v[e] += held[e];
                store4(p.out, 1, m * p.out_ld + n, left, vec, v);
            } else if constexpr (OUT == kPartial) {
                store4(p.out, 1, (part * p.m + m) * p.out_ld + n, left, vec, v);
            } else if constexpr (OUT == kGatePartial) {
                store4(p.out, 1, (part * 2 * p.m + m) * p.out_ld + n, left, vec, v);
                store4(p.out, 1, ((part * 2 + 1) * p.m + m) * p.out_ld + n, left, vec, acc[i][NF / 2 + j]);
            } else if constexpr (OUT == kTwoRows) {
                const bool first = m < p.half_rows;
                store4(first ? p.out : p.out2, 0, (first ? m : m - p.half_rows) * p.out_ld + n, left, vec, v);
            } else {
                constexpr int H = HALF ? NF / 2 : 0;
                const f32x4 u = acc[i][H + j];
                f32x4 h;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = silu(v[e]) * u[e];
                store4(p.out, 0, m * p.out_ld + n, left, vec, h);
                if (p.out2) {
                    store4(p.out2, 0, m * p.out_ld + n, left, vec, v);
                    store4(p.out3, 0, m * p.out_ld + n, left, vec, u);
                }
            }
        }
    }
}

}  // namespace tile_product
