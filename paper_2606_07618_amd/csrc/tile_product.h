// Tiled matrix product on the matrix cores of gfx950, D[m][n] = sum_k A[m][k] B[n][k], sums in
// binary32, for bfloat16 operands and for microscaled FP4 ones (E2M1 nibbles with an E8M0 scale
// for each 32 values of a row).  The kernels built from it differ in where their operands lie and
// in what is done with the sums; both are template arguments.
//
// Both element types share one geometry: a step takes 128 bytes of every row of the tile (64
// bfloat16 values, 256 FP4 ones), and a lane's operand of one matrix instruction is 16 of them (8
// values of 32x32x16, 32 of 32x32x64), so staging, LDS layout and register tiles are the same.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace tile_product {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kLanes = 64;
constexpr int kStepBytes = 128;                  // of a row, a step of the contraction
constexpr int kQuarters = kStepBytes / 32;      // matrix instructions a step along the contraction
constexpr int kChunk = 16;                       // bytes of a lane's load
constexpr uint32_t kOutside = 0x80000000u;       // an offset that the buffer's size excludes: reads as zero

// A window of 2 GiB from `base`: loads at offsets of kOutside and up return zero without an access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)kOutside, 0x00020000);
}

template <int V> struct Const { static constexpr int value = V; };

enum Kind { kBf16, kMx };
// How an operand lies in memory: its rows hold the contraction (kAlong), or the contraction runs down
// its rows and a row holds the operand's outer index (kAcross; bfloat16 only).
enum Layout { kAlong, kAcross };

struct Operand {
    const char* p;              // element (0, 0)
    const char* p2;             // the second matrix of a pair (see Pair)
    int64_t ld;                 // bytes from row to row
    const uint8_t* scales;      // microscaled: E8M0 codes [outer, scale_ld]
    int64_t scale_ld;
};

// Where operand B is two matrices.  kPairOuter: the tile's outer indexes are taken half from each, so
// that both products of one output meet in one lane.  kPairInner: the contraction runs over the first,
// then over the second.
enum Pair { kSingle, kPairOuter, kPairInner };

__device__ __forceinline__ float silu(float g) {
    // g / (1 + e^-g): e^-g overflows to infinity below -88, where the quotient's reciprocal is zero.
    const float e = __builtin_amdgcn_exp2f(g * -1.44269504f);
    return g * __builtin_amdgcn_rcpf(1.0f + e);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
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
template <Kind KIND, Layout LAYOUT, int R, int THREADS, bool HALF>
struct Side {
    static_assert(LAYOUT == kAlong || KIND == kBf16, "microscaled operands lie along their rows");
    static constexpr int kBytes = R * kStepBytes;
    static constexpr int kLoads = kBytes / (THREADS * kChunk);
    static_assert(kBytes % (THREADS * kChunk) == 0, "whole loads");
    static constexpr int kRowChunks = LAYOUT == kAlong ? kStepBytes / kChunk : R / 8;
    // what a step takes of the contraction: bytes of a row, or rows
    static constexpr int kFull = LAYOUT == kAlong ? kStepBytes : kStepBytes / 2;

    // LDS holds a step as rows of chunks.  A chunk's place in its row is exchanged by the row, so that
    // the lanes of a read hit all banks: along, 16 lanes read one chunk of 16 rows, and the row's
    // parity and the exchanged place cover the 256 bytes of the banks; across, 32 lanes read four
    // contraction rows by 64 bytes, and the place of a 64-byte unit is exchanged by those rows.
    __device__ static __forceinline__ int exchange(int row) {
        if constexpr (LAYOUT == kAlong) return (row >> 1) & 7;
        constexpr int kUnits = R / 32 < 4 ? R / 32 : 4;
        return (row & (kUnits - 1)) << 2;
    }

    uint32_t offset[kLoads];             // of this thread's loads from the step's base

    // left: the outer indexes from the tile's first one on.  With HALF, rows from R / 2 on are the same
    // outer indexes of the second matrix.
    __device__ __forceinline__ void init(int64_t left, int64_t ld, int tid) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = i * THREADS + tid, row = id / kRowChunks;
            const int chunk = (id % kRowChunks) ^ exchange(row);
            const int r = HALF ? row % (R / 2) : row;
            const bool in = LAYOUT == kAlong ? r < left : chunk * 8 < left;
            offset[i] = in ? (uint32_t)r * (uint32_t)ld + chunk * kChunk : kOutside;
        }
    }

    // Starts the loads of one step into LDS.  ahead: what is left of the contraction from the step's
    // first value on, in units of kFull; beyond it LDS gets zeros.
    __device__ __forceinline__ void load(const char* base, const char* base2, char* lds, int64_t ahead, int tid,
                                         int wave) const {
        const __amdgpu_buffer_rsrc_t w = window(base), w2 = HALF ? window(base2) : w;
        const int left = ahead > kFull ? kFull : ahead > 0 ? (int)ahead : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool second = HALF && i * THREADS / kRowChunks >= R / 2;
            const int id = i * THREADS + tid, row = id / kRowChunks;
            const int at = LAYOUT == kAlong ? ((id % kRowChunks) ^ exchange(row)) * kChunk : row;
            const uint32_t off = at < left ? offset[i] : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? w2 : w,
                                                     (lds_void*)(lds + (i * THREADS + wave * kLanes) * kChunk), kChunk,
                                                     (int)off, 0, 0, 0);
        }
    }

    // This lane's 16 bytes of the operand at outer indexes row0 .. row0 + 31 of the tile, quarter Q of the step.
    // bfloat16: values 16 Q + 8 (lane / 32) on.  Microscaled: the 32-value block 4 (lane / 32) + Q, so that the
    // quarters' scales are the bytes of one word.
    template <int Q>
    __device__ static __forceinline__ i32x4 read(const char* lds, int row0, int lane) {
        const int g = lane / 32;
        if constexpr (LAYOUT == kAlong) {
            const int row = row0 + lane % 32, chunk = KIND == kMx ? kQuarters * g + Q : 2 * Q + g;
            return *reinterpret_cast<const i32x4*>(lds + row * kStepBytes + ((chunk ^ exchange(row)) * kChunk));
        } else {
            // ds_read_b64_tr_b16: 16 lanes read four rows of 16 values, four each, and get a column each
            const int i = lane % 16, row = 16 * Q + 8 * g + (i >> 2);
            const int chunk = (row0 / 8 + lane / 16 % 2 * 2 + ((i & 3) >> 1)) ^ exchange(row);
            const char* at = lds + row * (R * 2) + chunk * kChunk + (i & 1) * 8;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * R * 2));
            return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Workgroup tile M_ x N_ by WM x WN waves.
template <int M_, int N_, int WM_, int WN_, int SLOTS = 2>
struct Tile {
    static constexpr int kSlots = SLOTS;                             // steps of the contraction in LDS
    static constexpr int M = M_, N = N_, WM = WM_, WN = WN_, kThreads = WM_ * WN_ * kLanes;
    static constexpr int kWavesPerSimd = M_ * N_ / (WM_ * WN_) > 8192 ? 1 : 2;   // 512 or 256 registers
    static constexpr int MF = M_ / WM_ / 32, NF = N_ / WN_ / 32;     // a wave's matrix instructions
};

// What happens to the sums.
enum Out {
    kSums,        // scale * sum, as bfloat16 or binary32
    kPartial,     // the sum of this part of the contraction, binary32, for a later reduction
    kGate,        // silu(sum of the first matrix) * sum of the second, and both sums where asked for
    kTwoRows      // rows below `half_rows` to the first output, those from there on to the second
};

struct Args {
    Operand a, b;
    int64_t m, n;               // outer indexes of A and of B (kPairOuter: of each of B's two)
    int64_t inner;              // values of the contraction (kPairInner: of each of B's two)
    int64_t steps, split_steps; // of the whole contraction, and of one part of it
    int64_t tiles_m, tiles_n;
    int parts;
    int out_f32;
    const float* scale;         // NULL: 1
    void *out, *out2, *out3;
    int64_t half_rows, out_rows;   // kTwoRows
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

template <Kind KIND, Layout LA, Layout LB, Pair PAIR, Out OUT, class T>
__global__ __launch_bounds__(T::kThreads, T::kWavesPerSimd) void product_kernel(Args p) {
    constexpr bool HALF = PAIR == kPairOuter;
    using A = Side<KIND, LA, T::M, T::kThreads, false>;
    using B = Side<KIND, LB, T::N, T::kThreads, HALF>;
    constexpr int kScales = KIND == kMx ? (T::M + T::N) * 2 * kQuarters : 0;   // eight bytes a row and step
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
    // the scales of A's rows, then of B's; a load is of one operand's rows
    uint32_t scale_offset[kScaleLoads + 1];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int row = (i * T::kThreads + tid) / 2, rb = row - T::M, word = tid % 2 * 4;
        scale_offset[i] = row < T::M ? (row < p.m - m0 ? (uint32_t)row * (uint32_t)p.a.scale_ld + word : kOutside)
                                     : (rb < p.n - n0 ? (uint32_t)rb * (uint32_t)p.b.scale_ld + word : kOutside);
    }
    const char* a0 = p.a.p + (LA == kAlong ? m0 * p.a.ld : m0 * 2);
    const int64_t b_at = LB == kAlong ? n0 * p.b.ld : n0 * 2;
    const int64_t pair_steps = PAIR == kPairInner ? p.steps / 2 : p.steps;
    auto fetch_a = [&](int64_t s, int stage) {
        const int64_t in = LA == kAlong ? (KIND == kMx ? p.inner / 2 : p.inner * 2) : p.inner;
        // kPairInner: A's rows hold both contractions one after the other, each filled up with zeros
        const int64_t ahead = PAIR == kPairInner ? (p.steps - s) * A::kFull : in - s * A::kFull;
        sa.load(a0 + (LA == kAlong ? s * kStepBytes : s * A::kFull * p.a.ld), nullptr, lds[stage], ahead, tid, wave);
    };
    auto fetch_b = [&](int64_t s, int stage) {
        char* l = lds[stage] + A::kBytes;
        const int64_t in = LB == kAlong ? (KIND == kMx ? p.inner / 2 : p.inner * 2) : p.inner;
        const bool second = PAIR == kPairInner && s >= pair_steps;
        const int64_t at = second ? s - pair_steps : s;
        const int64_t step = b_at + (LB == kAlong ? at * kStepBytes : at * B::kFull * p.b.ld);
        sb.load((second ? p.b.p2 : p.b.p) + step, HALF ? p.b.p2 + step : nullptr, l, in - at * B::kFull, tid, wave);
        if constexpr (KIND == kMx) {
            const bool any = p.inner / 32 - s * 8 > tid % 2 * 4;
            const __amdgpu_buffer_rsrc_t ra = window(p.a.scales + m0 * p.a.scale_ld + s * 8),
                                         rb = window(p.b.scales + n0 * p.b.scale_ld + s * 8);
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i) {
                const int first = i * T::kThreads + wave * kLanes;
                if (!kEven && first * 4 >= kScales) break;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(first / 2 < T::M ? ra : rb, (lds_void*)(l + B::kBytes + first * 4), 4,
                                                         (int)(any ? scale_offset[i] : kOutside), 0, 0, 0);
            }
        }
    };

    // first rows of this wave's fragments in the tile
    auto a_row = [&](int i) { return wm * (T::M / T::WM) + i * 32; };
    auto b_row = [&](int j) {
        if constexpr (!HALF) return wn * (T::N / T::WN) + j * 32;
        return (j < NF / 2 ? 0 : T::N / 2) + wn * (T::N / 2 / T::WN) + j % (NF / 2) * 32;
    };

    f32x16 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // Registers run a quarter of a step ahead of the matrix instructions, LDS kSlots steps: while one
    // quarter's fragments are multiplied the next one's are read, and the one barrier of a step stands
    // where its last fragments have been read, so that its LDS is free for the step kSlots on.  That step's
    // loads are started in two parts, A's behind the barrier and B's a quarter later, among the matrix
    // instructions: in one burst they fill the queue that both waves of a SIMD then wait at ([4096, 14336] x
    // [14336, 4096], contraction down the rows: 487 -> 449 us).  What a step waits for at its barrier are
    // the loads of the next step, and no later ones.
    i32x4 fa[2][MF], fb[2][NF];
    int xa[2][MF], xb[2][NF];                  // scales of this step and of the next
    auto read = [&](auto q, int stage) {
        constexpr int Q = decltype(q)::value;
        const char* la = lds[stage];
        const char* lb = la + A::kBytes;
#pragma unroll
        for (int j = 0; j < NF; ++j) fb[Q % 2][j] = B::template read<Q>(lb, b_row(j), lane);
#pragma unroll
        for (int i = 0; i < MF; ++i) fa[Q % 2][i] = A::template read<Q>(la, a_row(i), lane);
        if constexpr (KIND == kMx && Q == 0) {
            const char* ls = lb + B::kBytes + lane / 32 * 4;
#pragma unroll
            for (int j = 0; j < NF; ++j)
                xb[1][j] = *reinterpret_cast<const int*>(ls + (T::M + b_row(j) + lane % 32) * 8);
#pragma unroll
            for (int i = 0; i < MF; ++i)
                xa[1][i] = *reinterpret_cast<const int*>(ls + (a_row(i) + lane % 32) * 8);
        }
    };
    auto multiply = [&](auto q) {
        constexpr int Q = decltype(q)::value;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                // B's values as the instruction's rows: a lane gets runs of four neighbouring outputs of a row of D
                const i32x4 b = fb[Q % 2][j], a = fa[Q % 2][i];
                if constexpr (KIND == kBf16) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b),
                                                                        __builtin_bit_cast(bf16x8, a), acc[i][j], 0, 0, 0);
                } else {
                    const i32x8 wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0}, wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wb, wa, acc[i][j], 4, 4, Q, xb[0][j], Q,
                                                                                xa[0][i]);
                }
            }
        }
    };
    // the LDS reads of a quarter, and the loads it starts, spread among the matrix instructions of the one before
    auto interleave = [&](int loads) {
        constexpr int kReads = MF * (LA == kAcross ? 2 : 1) + NF * (LB == kAcross ? 2 : 1), kOps = MF * NF;
        constexpr int kEach = kReads > kOps ? (kReads + kOps - 1) / kOps : 1;
#pragma unroll
        for (int r = 0; r < kOps; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);               // LDS reads
            if (r < loads) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);    // loads from memory
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                   // matrix instructions
        }
    };
    auto next_scales = [&]() {
        if constexpr (KIND == kMx) {
#pragma unroll
            for (int i = 0; i < MF; ++i) xa[0][i] = xa[1][i];
#pragma unroll
            for (int j = 0; j < NF; ++j) xb[0][j] = xb[1][j];
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
        read(Const<0>{}, 0);
        int slot = 0;
        for (int64_t s = s0; s < s1; ++s) {
            const int next = slot + 1 == kSlots ? 0 : slot + 1;
            next_scales();
            read(Const<1>{}, slot);
            if (s > s0) fetch_b(s - 1 + kSlots, slot == 0 ? kSlots - 1 : slot - 1);
            multiply(Const<0>{});
            interleave(B::kLoads);
            read(Const<2>{}, slot);
            multiply(Const<1>{});
            interleave(0);
            read(Const<3>{}, slot);
            multiply(Const<2>{});
            interleave(0);
            arrive<(kSlots - 2) * kLoads>();
            fetch_a(s + kSlots, slot);
            read(Const<0>{}, next);
            multiply(Const<3>{});
            interleave(A::kLoads);
            slot = next;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // no load into LDS outlives the workgroup
    }

    // a lane holds, of row lane % 32 of D, the runs of four columns from 4 (lane / 32) on, eight apart
    const bool vec = p.out_ld % 4 == 0;
    const float scale = OUT == kSums && p.scale ? *p.scale : 1.0f;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t m = m0 + a_row(i) + lane % 32;
        if (m >= p.m) continue;
#pragma unroll
        for (int jr = 0; jr < (HALF ? NF / 2 : NF) * 4; ++jr) {
            const int j = jr / 4, r = jr % 4 * 4;
            const int64_t n = n0 + b_row(j) + r * 2 + lane / 32 * 4, left = p.n - n;
            const f32x4 v = {acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]};
            if constexpr (OUT == kSums) {
                store4(p.out, p.out_f32, m * p.out_ld + n, left, vec, v * scale);
            } else if constexpr (OUT == kPartial) {
                store4(p.out, 1, (part * p.m + m) * p.out_ld + n, left, vec, v);
            } else if constexpr (OUT == kTwoRows) {
                const int64_t row = m < p.half_rows ? m : m - p.half_rows;
                if (row < p.out_rows)
                    store4(m < p.half_rows ? p.out : p.out2, 0, row * p.out_ld + n, left, vec, v);
            } else {
                constexpr int H = HALF ? NF / 2 : 0;
                const f32x4 u = {acc[i][H + j][r], acc[i][H + j][r + 1], acc[i][H + j][r + 2], acc[i][H + j][r + 3]};
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
