// Products of rows sorted by group (the tokens of each expert) with the NVFP4 weights of their own group.  Where a
// group's rows begin is known on the device alone, so a workgroup finds its rows itself: tiles are numbered through all
// groups, and each wave sums the groups' tile counts up to its own number.
//
//   y[i][n]  = S_e sum_k x[i][k] (q s)_e[n][k]      weights as they lie: the contraction runs along their rows
//   dx[i][k] = S_e sum_n dy[i][n] (q s)_e[n][k]     turned: it runs down their rows
//
// A weight q s has six significant bits and is exact in bfloat16, the type of the rows; sums are binary32.
#pragma once

#include "grouped_plan.h"
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

// Where a row tile lies: its expert, its rows first .. first + left - 1 (left: to the group's end).
struct Place { int expert; int64_t first, left; };
// All groups: their row tiles, and their rows begin .. end - 1.
struct Groups { int tiles, begin, end; };

__device__ __forceinline__ int at_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// The sum, or the largest, of this lane's value and those of the lanes before it; values are not negative.
template <int CTRL, int ROWS, bool SUM>
__device__ __forceinline__ int scan_step(int v) {
    const int o = __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, true);
    return SUM ? v + o : v > o ? v : o;
}
template <bool SUM>
__device__ __forceinline__ int scan(int v) {
    v = scan_step<0x111, 0xF, SUM>(v);           // within rows of 16: 1, 2, 4, 8 lanes before
    v = scan_step<0x112, 0xF, SUM>(v);
    v = scan_step<0x114, 0xF, SUM>(v);
    v = scan_step<0x118, 0xF, SUM>(v);
    v = scan_step<0x142, 0xA, SUM>(v);           // rows 1 and 3: the last lane of the row before
    return scan_step<0x143, 0xC, SUM>(v);        // rows 2 and 3: lane 31
}

// What every look at the groups begins with: offsets[0], and offsets[lane + 1].
struct Offsets { int zero, next; };
__device__ __forceinline__ Offsets offsets_of(const Args& p, int lane) {
    return {p.offsets[0], lane < p.experts ? p.offsets[lane + 1] : 0};
}

// Goes through the groups, a wave's lanes 64 at a time: each(first group, a lane's tiles, tiles up to it and with it, its
// first row, its end) until that says true.  Offsets are taken within 0 .. rows and never descend: what does not fit makes
// a group shorter or empty.
template <class Each>
__device__ __forceinline__ Groups through(const Args& p, Offsets o, int height, int lane, Each each) {
    const int rows = (int)p.rows;
    auto within = [&](int v) { return v < 0 ? 0 : v > rows ? rows : v; };
    auto end_of = [&](int e) { return e < p.experts ? p.offsets[e + 1] : 0; };
    int next = o.next, before = within(o.zero), total = 0;
    const int begin = before;
    for (int base = 0; base < p.experts; base += kLanes) {
        int end = scan<false>(within(next));     // past the last expert: as the last one's
        next = end_of(base + kLanes + lane);
        if (end < before) end = before;
        int start = __shfl_up(end, 1);
        if (lane == 0) start = before;
        const int tiles = (int)((end - start + (int64_t)height - 1) / height), upto = scan<true>(tiles);
        if (each(base, total, tiles, upto, start, end)) break;
        total += at_lane(upto, kLanes - 1);      // tiles are fewer than 2^31
        before = at_lane(end, kLanes - 1);
    }
    return {total, begin, before};
}

__device__ __forceinline__ Groups groups_of(const Args& p, Offsets o, int height, int lane) {
    return through(p, o, height, lane, [](int, int, int, int, int, int) { return false; });
}

// Row tile `index` of those that there are.
__device__ __forceinline__ Place place_of(const Args& p, Offsets o, int index, int height, int lane) {
    Place t = {0, 0, 0};
    through(p, o, height, lane, [&](int base, int total, int tiles, int upto, int start, int end) {
        const uint64_t mine = __ballot(index - total < upto);
        if (!mine) return false;
        const int l = __builtin_ctzll(mine), s = at_lane(start, l);
        const int64_t first = s + (int64_t)(index - total - at_lane(upto - tiles, l)) * height;
        t = {base + l, first, at_lane(end, l) - first};
        return true;
    });
    return t;
}

// What a workgroup does.  An XCD gets a run of the sequence of tiles, which walks kDeep row tiles at a time, so that what
// it works on at one time shares rows and weights in its L2.  Where an XCD's last tiles would keep few of its compute
// units busy (SPLIT, one workgroup each), they are cut into two or four parts of their rows ([8192, 14336] x eight times
// [14336, 4096], 72 tiles for 32 units: 957 us, 1082 without).  The workgroups that are over: `spare` of `sharers`.
using grouped_plan::kUnits, grouped_plan::kFewThreads;
constexpr int kDeep = 8;
struct Work { bool tile; int index; int64_t n; int part, parts; int64_t spare, sharers; };
template <bool SPLIT>
__device__ __forceinline__ Work work_of(int64_t id, int64_t launched, int tiles_m, int64_t tiles_n) {
    const int64_t count = tiles_m * tiles_n, xcd = id % kXcds, local = id / kXcds;
    const int64_t each = count / kXcds, rest = count % kXcds, mine = each + (xcd < rest), last = SPLIT ? mine % kUnits : 0, whole = mine - last;
    const int parts = last <= kUnits / 4 ? 4 : last <= kUnits / 2 ? 2 : 1;
    const int64_t used = whole + last * parts;
    if (local >= used) return {false, 0, 0, 0, 0, (local - used) * kXcds + xcd, (launched / kXcds - used) * kXcds};
    const bool cut = local >= whole;
    const int64_t in_run = cut ? whole + (local - whole) / parts : local;
    const int64_t seq = xcd * each + (xcd < rest ? xcd : rest) + in_run;
    const int64_t first = seq / (kDeep * tiles_n) * kDeep, height = tiles_m - first < kDeep ? tiles_m - first : kDeep;
    const int64_t in = seq % (kDeep * tiles_n);
    return {true, (int)(first + in % height), in / height, cut ? (int)((local - whole) % parts) : 0, cut ? parts : 1, 0, 0};
}

// Rows of no group: the workgroups that have no tile share them out.
__device__ __forceinline__ void clear_rows(const Args& p, const Groups& all, const Work& w, int tid, int threads) {
    if (!p.clear) return;
    for (int64_t i = w.spare; i < all.begin + (p.rows - all.end); i += w.sharers) {
        const int64_t m = i < all.begin ? i : all.end + (i - all.begin);
        for (int64_t n = tid; n < p.outer; n += threads) {
            if (p.out_f32) static_cast<float*>(p.out)[m * p.outer + n] = 0.0f;
            else static_cast<uint16_t*>(p.out)[m * p.outer + n] = 0;
        }
    }
}

// ---- weights and scales by groups of 256 values of a row ------------------------------------------

// A window of at most 2 GiB over the `left` bytes from `base` on: loads past it return zero without an access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window_of(const void* base, int64_t left) {
    // by halves, in scalar registers
    const uint32_t high = (uint32_t)((uint64_t)left >> 32), low = (uint32_t)left, most = low < kOutside ? low : kOutside;
    const uint32_t size = high == 0 ? most : (int)high < 0 ? 0u : kOutside;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)size, 0x00020000);
}

// Stores to LDS that wait for nothing: as ordinary ones they would wait for all LDS loads on their way, which go to other
// places (the compiler cannot know).  arrive() waits for them.  at: an address in LDS.
template <int OFFSET>
__device__ __forceinline__ void put8(uint32_t at, i32x2 v) { asm volatile("ds_write_b64 %0, %1 offset:%2" ::"v"(at), "v"(v), "n"(OFFSET)); }

// The scales of a group of N rows, 16 bytes a row at most, by two threads a row: as words where rows of them are whole words,
// else one by one.
template <int N>
struct GroupScales {
    const uint8_t* from;
    int64_t left;
    uint32_t at;
    int each, half;                              // of a row and group; of it, this thread's first
    bool words;
    __device__ __forceinline__ void init(const Args& p, int64_t w_row, int64_t n0, int tid) {
        const int64_t ld = p.k >> p.shift;
        from = p.scales + w_row * ld, left = (p.n - n0) * ld;
        each = 256 >> p.shift, half = tid % 2 * 8;
        at = tid < 2 * N && n0 + tid / 2 < p.n ? (uint32_t)(tid / 2) * (uint32_t)ld + half : kOutside;
        words = ((each | (int)ld | (int)(uintptr_t)p.scales) & 3) == 0;
    }
    __device__ __forceinline__ i32x2 load(int group) const {
        const int64_t done = (int64_t)group * each;
        const __amdgpu_buffer_rsrc_t w = window_of(from + done, left - done);
        if (words) return load8(w, at);
        uint32_t c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = load1(w, half + i < each ? at + i : kOutside);
        return i32x2{(int)(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24), (int)(c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24)};
    }
};

// Rows of 128 bytes in LDS, loaded as Side's but for their exchange: a lane of a fragment reads chunk 2 (lane / 16) or the
// one behind it, and of the lanes that LDS serves at once rows 0 to 3 and 12 to 15 are from one sixteen, rows 4 to 11 from the
// next, two chunks on.  The places of these two sets of rows are apart from each other, moved by two or not.  (With Side's
// exchange conflicts are half of LDS' time, 0.22 of it so; 16384 rows, eight groups, [14336, 4096] take 1.58 ms either way, held by
// the power limit.)
template <int R, int THREADS>
struct Rows {
    static constexpr int kLoads = R * kStepBytes / (THREADS * kChunk);
    static_assert(THREADS / 8 % 16 == 0 && kLoads * THREADS * kChunk == R * kStepBytes, "a thread's rows have one exchange");
    __device__ static __forceinline__ int exchange(int row) {
        const int i = row >> 1 & 7;
        return ((i >> 2 ^ i >> 1) & 1) << 2 | (i >> 2) << 1 | (i & 1);
    }
    uint32_t offset[kLoads];
    int at;                                      // of this thread's chunk in a row
    __device__ __forceinline__ void init(int64_t left, int64_t ld, int tid) {
        at = (tid % 8 ^ exchange(tid / 8)) * kChunk;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = (i * THREADS + tid) / 8;
            offset[i] = row < left ? (uint32_t)row * (uint32_t)ld + at : kOutside;
        }
    }
    __device__ __forceinline__ void load(const char* base, char* lds, int64_t ahead, int wave) const {
        const __amdgpu_buffer_rsrc_t w = window(base);
        const int left = ahead > kStepBytes ? kStepBytes : ahead > 0 ? (int)ahead : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w, (lds_void*)(lds + (i * THREADS + wave * kLanes) * kChunk), kChunk,
                                                     (int)(at < left ? offset[i] : kOutside), 0, 0, 0);
    }
};

// ---- few rows a group ---------------------------------------------------------------------------
// Reading the weights is all there is to do.  A workgroup owns 64 R weight rows, 16 R for each of four waves, and up to 16 C
// rows of one group; weights, scales and rows go through LDS by whole lines, 256 values of the contraction at a time, the next
// ones while these are multiplied.  512 rows, 128 groups, [1536, 4096]: 103 us, 4.5 TB/s, where a large copy reaches 5.1 and a large
// read 6.2; a tenth of the bytes are the scales, 16 bytes of a row at a time.  Three workgroups a compute unit hide each other's first waits;
// rings of three or four stages leave room for two (an eighth longer).  Loaded straight into the registers of
// the matrix instructions, whose neighbouring lanes hold different rows, each lane's 16 bytes are an access of their own to the
// L1, which was then nine tenths of the time busy (a fifth longer).
// H: fours of waves that take turns along the contraction, whose sums meet in LDS at the end: where workgroups are few, a
// stage's way from LDS through the matrix instructions is what there is to wait for (two rows of eight groups, [14336, 4096]:
// 19.4 us with two fours, 21.1 with one, 24.0 with four).
template <int R, int C, int H>
__global__ __launch_bounds__(kFewThreads * H, 2) void few_kernel(Args p) {
    constexpr int N = 64 * R, kRows = 16 * C, kW = N * kStepBytes, kX = kRows * 512, kS = N * 16, kStage = kW + kX + kS;
    using B = Rows<N, kFewThreads>;
    constexpr int kXLoads = kX / (kFewThreads * kChunk);
    __shared__ __attribute__((aligned(1024))) char lds_of[H][2 * kStage];
    static_assert((H - 1) * kFewThreads * R * C * sizeof(f32x4) <= sizeof(lds_of), "the other part's sums");
    const int part = H > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kFewThreads) : 0;   // of the contraction's stages, every H-th
    const int tid = threadIdx.x % kFewThreads, lane = tid % kLanes, g = lane / 16, l16 = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    char* lds = lds_of[part];
    const Offsets offsets = offsets_of(p, lane);
    const Groups all = groups_of(p, offsets, kRows, lane);
    const Work work = work_of<false>(blockIdx.x, gridDim.x, all.tiles, p.tiles_n);
    if (!work.tile) return clear_rows(p, all, work, threadIdx.x, kFewThreads * H);
    const int64_t n0 = work.n * N;
    const Place t = place_of(p, offsets, work.index, kRows, lane);

    const float S = p.S[t.expert];
    const int64_t q_ld = p.k / 2, w_row = t.expert * p.n + n0, q_left = (p.n - n0) * q_ld, x_bytes = p.k * 2;
    const char *q0 = p.q + w_row * q_ld, *x0 = p.x + t.first * p.ld;
    B sb;
    sb.init(p.n - n0, q_ld, tid);
    GroupScales<N> scales_of;
    scales_of.init(p, w_row, n0, tid);
    // 32 chunks of a row of x, their places exchanged by the row, as Rows' are for chunks eight apart
    auto place = [](int row) { return (row & 8) | ((row >> 3 ^ row >> 2) & 1) << 2 | (row & 3); };
    uint32_t x_at[kXLoads];
    const int x_chunk = tid % 32;
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
        const int row = (i * kFewThreads + tid) / 32;
        x_at[i] = row < t.left ? (uint32_t)row * (uint32_t)p.ld + (x_chunk ^ place(row)) * kChunk : kOutside;
    }
    i32x2 scales[2];
    auto fetch = [&](int turn, auto dc) {
        constexpr int d = decltype(dc)::value;
        const int s = turn * H + part;
        char* to = lds + d * kStage;
        // A row's last chunk may hold the next row's first values, finite numbers: they meet zeros.
        const int64_t done = (int64_t)s * kStepBytes, x_done = (int64_t)s * 512, q_ahead = q_ld - done, x_ahead = x_bytes - x_done;
        const int q_in = q_ahead > kStepBytes ? kStepBytes : q_ahead > 0 ? (int)q_ahead : 0, x_in = x_ahead > 512 ? 512 : x_ahead > 0 ? (int)x_ahead : 0;
        const __amdgpu_buffer_rsrc_t rq = window_of(q0 + done, q_left - done), rx = window(x0 + x_done);
#pragma unroll
        for (int i = 0; i < B::kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_void*)(to + (i * kFewThreads + wave * kLanes) * kChunk), kChunk,
                                                     (int)(sb.at < q_in ? sb.offset[i] : kOutside), 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            const int at = (x_chunk ^ place((i * kFewThreads + tid) / 32)) * kChunk;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void*)(to + kW + (i * kFewThreads + wave * kLanes) * kChunk), kChunk,
                                                     (int)(at < x_in ? x_at[i] : kOutside), 0, 0, 0);
        }
        scales[d] = scales_of.load(s);
    };

    f32x4 acc[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) acc[r][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // A lane takes 64 neighbouring values of its row, chunks 2 g and 2 g + 1 of a stage's weights, under four scales at most.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
    const int w_row0 = wave * (16 * R) + l16;
    auto compute = [&](auto dc) {
        constexpr int d = decltype(dc)::value;
        const char *w = lds + d * kStage, *x = w + kW, *c = x + kX;
        uint32_t s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = w_row0 + r * 16;
            s[r] = *reinterpret_cast<const uint32_t*>(c + row * 16 + ((4 * g) >> (p.shift - 4) & ~3));
            if (p.shift > 4) s[r] >>= ((4 * g) >> (p.shift - 4)) % 4 * 8;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 wv[R], xv[C][4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int row = w_row0 + r * 16;
                wv[r] = *reinterpret_cast<const i32x4*>(w + row * kStepBytes + ((2 * g + h) ^ B::exchange(l16)) * kChunk);
            }
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    xv[i][j] = *reinterpret_cast<const i32x4*>(x + (i * 16 + l16) * 512 + ((8 * g + 4 * h + j) ^ place(l16)) * kChunk);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                // blocks of 16: a scale for two of the four; of 32: for all four; of more: the same for both halves
                const uint32_t c0 = p.shift == 4 ? s[r] >> 16 * h : p.shift == 5 ? s[r] >> 8 * h : s[r], c1 = p.shift == 4 ? c0 >> 8 : c0;
                const float f0 = e4m3_f32(c0), f1 = e4m3_f32(c1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 v = expand8((uint32_t)wv[r][j], j < 2 ? f0 : f1);
#pragma unroll
                    for (int i = 0; i < C; ++i)
                        acc[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, xv[i][j]), acc[r][i], 0, 0, 0);
                }
            }
        }
    };
    const int turns = (int)((p.k + 256 * H - 1) / (256 * H));   // past the last stage: zeros
    auto stage = [&](int s, auto dc) {
        constexpr int d = decltype(dc)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (tid < 2 * N) put8<0>(lds0 + d * kStage + kW + kX + tid * 8, scales[d]);
        arrive<0>();
        fetch(s + 1, Const<1 - d>{});            // where the last stage was
        compute(dc);
    };
    fetch(0, Const<0>{});
    for (int s = 0; s < turns; s += 2) {
        stage(s, Const<0>{});
        if (s + 1 < turns) stage(s + 1, Const<1>{});
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load into LDS outlives the workgroup
    if constexpr (H > 1) {
        __syncthreads();
        f32x4* sums = reinterpret_cast<f32x4*>(lds_of[0]);
        if (part > 0) {
#pragma unroll
            for (int f = 0; f < R * C; ++f) sums[((part - 1) * R * C + f) * kFewThreads + tid] = acc[f / C][f % C];
        }
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int o = 0; o < H - 1; ++o)
#pragma unroll
            for (int f = 0; f < R * C; ++f) acc[f / C][f % C] += sums[(o * R * C + f) * kFewThreads + tid];
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < C; ++i) {
            // a lane holds outputs n .. n + 3 of a row
            const int64_t n = n0 + wave * (16 * R) + r * 16 + g * 4, row = i * 16 + l16;
            if (row < t.left) store4(p.out, p.out_f32, (t.first + row) * p.outer + n, p.outer - n, p.outer % 4 == 0, acc[r][i] * S);
        }
}

// ---- tiles --------------------------------------------------------------------------------------
// 256 rows by 256 outputs, or 128 by 128, of one group; a group's last tile computes as many rows as it needs, in halves.  A
// step of the contraction is 64 values.  The rows go from memory straight into LDS, one step ahead.  Weights as they lie go
// there too, as nibbles, and each wave expands what it multiplies.  Turned ones are expanded by the threads that load them,
// once for a tile's rows, on their way into LDS, where they lie as bfloat16 rows along the contraction: turning costs nothing
// there, as the pairs that share a register are put together from single values anyway.
// 64 rows: each wave takes all of them against half as many weight rows, and so expands half as many, and the rows are four
// steps ahead (6400 rows, 128 groups, [1536, 4096]: 171 us; a seventh longer without either).
//   16384 rows, eight groups, [14336, 4096]: 1.58 ms (1.22 PFLOP/s; the clock is held below 1.8 GHz by the power limit,
//   and the matrix instructions are busy two thirds of a compute unit's time); turned, 8192 rows: 0.96 ms (1.00 PFLOP/s).
constexpr int kSteps = 2;                        // in LDS

// Turned weights: a row's chunks of 16 bytes exchanged by the row, as reads take one chunk of 16 neighbouring rows and
// writes one of rows 8 apart.
__device__ __forceinline__ int exchange(int row) { return ((row >> 1) ^ (row >> 4)) & 7; }

template <int M_, int WN_>
struct Tile {
    static constexpr int M = M_, WM = 2, WN = WN_, N = WN_ * 64, kThreads = WM * WN_ * kLanes;
    static constexpr int kStage = (M + N) * kStepBytes;              // of LDS, a step of rows and turned weights; a power of two
    static constexpr int kLds = kSteps * (kStage + N * 16);
    static constexpr bool kSplit = M_ == 256;                        // one workgroup a compute unit
    static constexpr int kMost = M_ / 32;                            // a wave's fragments of rows
};

// A thread's turned weights of a step, 8 columns of four rows, and where they lie from the step's first row on.  Past the
// group's weights they are zero.
template <class T>
struct Turned {
    static constexpr int kLoads = 8, kParts = 4;
    __device__ static __forceinline__ int column_of(int tid) { return tid % (T::N / 8) * 8; }
    __device__ static __forceinline__ int row_of(int tid) { return tid / (T::N / 8) * 4; }
    struct From {
        uint32_t q, s, q_ld, s_ld;
        __device__ __forceinline__ void init(const Args& p, int64_t n0, int tid) {
            q_ld = (uint32_t)(p.k / 2), s_ld = (uint32_t)(p.k >> p.shift);
            const int column = column_of(tid), row = row_of(tid);
            const bool in = n0 + column < p.k;
            q = in ? (uint32_t)row * q_ld + (uint32_t)column / 2 : kOutside;
            s = in ? (uint32_t)row * s_ld + (((uint32_t)n0 + column) >> p.shift) : kOutside;
        }
        __device__ __forceinline__ void remake() { asm volatile("" : "+v"(q), "+v"(s)); }
    };
    i32x4 v;
    uint32_t s[4];

    __device__ __forceinline__ void load(const From& at, __amdgpu_buffer_rsrc_t rq, __amdgpu_buffer_rsrc_t rs) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = __builtin_amdgcn_raw_buffer_load_b32(rq, (int)(at.q + r * at.q_ld), 0, 0);
            s[r] = load1(rs, at.s + r * at.s_ld);
        }
    }

    // Where a thread's weights go in LDS: with its chunks' places exchanged, column 2 Q + J lies at base ^ 16 Q, 256 Q + 128 J on.
    __device__ static __forceinline__ uint32_t base(int tid) {
        const int column = column_of(tid), row = row_of(tid);
        return column * kStepBytes + ((row / 8) ^ exchange(column)) * kChunk + row % 8 * 2;
    }
    // Part Q, two columns of the four rows, to LDS at base address `to`.
    template <int Q>
    __device__ __forceinline__ void store(uint32_t to) const {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[0], 1.0f, Q) * e4m3_f32(s[0]),
                    b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[1], 1.0f, Q) * e4m3_f32(s[1]),
                    c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[2], 1.0f, Q) * e4m3_f32(s[2]),
                    d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)v[3], 1.0f, Q) * e4m3_f32(s[3]);
        // the upper halves of the products hold all of them
        const auto pair = [](float lo, float hi) { return (int)__builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); };
        put8<2 * Q * kStepBytes>(to ^ (Q * kChunk), i32x2{pair(a[0], b[0]), pair(c[0], d[0])});
        put8<(2 * Q + 1) * kStepBytes>(to ^ (Q * kChunk), i32x2{pair(a[1], b[1]), pair(c[1], d[1])});
    }
};

// The sums of a tile, times the global scale, to the rows that there are.  All waves are done with LDS' contents.
template <class T, int MF, int NF>
__device__ __forceinline__ void finish(const Args& p, const Place& t, int64_t n0, char* lds, int tid, const f32x4 (&acc)[MF][NF]) {
    constexpr int WN = T::N / (NF * 16), kRows = MF * 16 * (T::kThreads / kLanes / WN);
    const int lane = tid % kLanes, wave = __builtin_amdgcn_readfirstlane(tid / kLanes), wm = wave / WN, wn = wave % WN;
    auto a_row = [&](int i) { return wm * (MF * 16) + i * 16; };
    auto b_row = [&](int j) { return (wn * NF + j) * 16; };
    const float S = p.S[t.expert];
    if (!p.out_f32 && p.outer % 8 == 0) {
        // through LDS, as whole rows of the tile
        constexpr int kOutChunks = T::N / 8, kMask = 15;
        static_assert(kRows * T::N * 2 <= T::kLds, "the tile in LDS");
        char* tile = lds;
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
            if (row < t.left && n < p.outer) {
                const i32x4 v = *reinterpret_cast<const i32x4*>(tile + (row * kOutChunks + (chunk ^ (row & kMask))) * kChunk);
                i32x4* to = reinterpret_cast<i32x4*>(static_cast<uint16_t*>(p.out) + (t.first + row) * p.outer + n);
                if constexpr (T::M == 256) __builtin_nontemporal_store(v, to);      // past the L2, which the operands need
                else *to = v;
            }
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

// The product of one tile with weights as they lie, MF fragments of 16 rows by NF of 16 weight rows a wave.
//
// Weights go into LDS as they are, 256 values of each row (whole lines) at a time, and from there into the registers of
// each wave, which expands the fragments that it multiplies, once for its 16 MF rows.  (Expanded once for the whole tile,
// as turned ones are, each weight is written to LDS, four times as wide: those stores took 0.45 of a step's 1.6 us, and
// expanding, twice as often so, fits between the matrix instructions.)
template <class T, int MF, int NF>
__device__ __forceinline__ void product_raw(const Args& p, const Place& t, int64_t n0, char* lds, int tid) {
    constexpr int WN = T::N / (NF * 16), kRows = MF * 16 * (T::kThreads / kLanes / WN), kA = kRows * kStepBytes, kB = T::N * kStepBytes, kS = T::N * 16;
    constexpr int kB0 = 2 * T::M * kStepBytes, kS0 = kB0 + 2 * kB;     // of LDS: rows, weights, scales, two of each
    constexpr int kSlots = kRows < T::M ? 4 : 2;            // of rows: fewer of them, whose steps are short, further ahead
    using A = Rows<kRows, T::kThreads>;
    using B = Side<T::N, T::kThreads, false>;              // 256 values in 128 bytes
    static_assert(B::kLoads == 4 && T::kThreads == 2 * T::N, "the loads' order");
    const int lane = tid % kLanes, wave = __builtin_amdgcn_readfirstlane(tid / kLanes), wm = wave / WN, wn = wave % WN;
    A sa;
    B sb;
    sa.init(t.left, p.ld, tid);
    const int64_t q_ld = p.k / 2, w_row = t.expert * p.n + n0;
    sb.init(p.n - n0, q_ld, tid);
    const char *a0 = p.x + t.first * p.ld, *q0 = p.q + w_row * q_ld;
    const int64_t q_left = (p.n - n0) * q_ld, row_bytes = p.k * 2;
    auto fetch_a = [&](int s, int slot) {
        sa.load(a0 + (int64_t)s * kStepBytes, lds + slot * kA, row_bytes - (int64_t)s * kStepBytes, wave);
    };
    // Half of a group's weights.  A row's last chunk may hold the next row's first values, finite numbers, which meet zeros;
    // behind the last row the window ends, and each word past it is zero.
    auto fetch_q = [&](int group, int slot, auto hc) {
        constexpr int H = decltype(hc)::value;
        const int64_t done = (int64_t)group * kStepBytes, ahead = q_ld - done;
        const int left = ahead > kStepBytes ? kStepBytes : ahead > 0 ? (int)ahead : 0;
        const __amdgpu_buffer_rsrc_t w = window_of(q0 + done, q_left - done);
#pragma unroll
        for (int i = 2 * H; i < 2 * H + 2; ++i) {
            const int row = (i * T::kThreads + tid) / 8, at = ((tid % 8) ^ B::exchange(row)) * kChunk;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w, (lds_void*)(lds + kB0 + slot * kB + (i * T::kThreads + wave * kLanes) * kChunk), kChunk,
                                                     (int)(at < left ? sb.offset[i] : kOutside), 0, 0, 0);
        }
    };
    GroupScales<T::N> scales_of;
    scales_of.init(p, w_row, n0, tid);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
    auto put_s = [&](i32x2 v, int slot) { put8<0>(lds0 + kS0 + slot * kS + tid * 8, v); };

    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // A lane of a fragment holds 16 values of a step, chunks 2 (lane / 16) and the one behind it of 8 values each, of its
    // row: the contraction's order does not matter as long as both operands have the same.  Chunks' places are exchanged by
    // their row.  Addresses are made in each step, not kept for all.
    const int l16 = lane % 16, g4 = lane / 16;
    struct {
        uint32_t a, b, c;
        __device__ __forceinline__ void remake() { asm volatile("" : "+v"(a), "+v"(b), "+v"(c)); }
    } at = {(uint32_t)((wm * (MF * 16) + l16) * kStepBytes + ((2 * g4) ^ A::exchange(l16)) * kChunk),
            (uint32_t)(kB0 + (wn * (NF * 16) + l16) * kStepBytes + ((g4 / 2) ^ B::exchange(l16)) * kChunk + g4 % 2 * 8),
            (uint32_t)(kS0 + (wn * (NF * 16) + l16) * 16)};
    const int down = p.shift - 4;

    // A step is 2 MF groups of NF matrix instructions.  While one half's are multiplied the other half's weights are
    // expanded: this step's second half, then the next step's first.
    constexpr int kParts = 2 * NF / MF;                    // halves of fragments that a group expands
    constexpr int kLead = MF >= 8 ? 3 : 2, kRing = 4, kGroups = 2 * MF;
    const int steps = (int)((p.k + 63) / 64);
    i32x4 fa[kRing], fb[2][NF];
    i32x2 raw[2][NF], scales = {0, 0};
    float f[2][NF];
    auto read_a = [&](auto gc, uint32_t from) {            // the fragment of group g of a step
        constexpr int g = decltype(gc)::value;
        fa[g % kRing] = *reinterpret_cast<const i32x4*>(lds + (from ^ (g / MF * kChunk)) + g % MF * (16 * kStepBytes));
    };
    auto read_b = [&](auto dc, auto uc, uint32_t slot) {   // step U of a group, to set D
        constexpr int D = decltype(dc)::value, U = decltype(uc)::value;
        const uint32_t c = at.c + (slot ? kS : 0) + ((4 * U + g4) >> down);
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            raw[D][j] = *reinterpret_cast<const i32x2*>(lds + ((at.b + (slot ? kB : 0)) ^ (U * 2 * kChunk)) + j * (16 * kStepBytes));
            f[D][j] = __uint_as_float(*reinterpret_cast<const uint8_t*>(lds + c + j * 256));
        }
    };
    auto scale_of = [&](auto dc) {
        constexpr int D = decltype(dc)::value;
#pragma unroll
        for (int j = 0; j < NF; ++j) f[D][j] = e4m3_f32(__float_as_uint(f[D][j]));
    };
    auto expand = [&](auto dc, auto hc, auto jc, auto pc) {    // four values: half P of fragment J's half H of set D
        constexpr int D = decltype(dc)::value, H = decltype(hc)::value, J = decltype(jc)::value, P = decltype(pc)::value;
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)raw[D][J][H], 1.0f, 2 * P) * f[D][J],
                    b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)raw[D][J][H], 1.0f, 2 * P + 1) * f[D][J];
        // the upper halves of the products hold all of them
        fb[H][J][2 * P] = (int)__builtin_amdgcn_perm(__float_as_uint(a[1]), __float_as_uint(a[0]), 0x07060302u);
        fb[H][J][2 * P + 1] = (int)__builtin_amdgcn_perm(__float_as_uint(b[1]), __float_as_uint(b[0]), 0x07060302u);
    };
    auto in_order = [] { asm volatile("" ::: "memory"); };   // the waits count on it
    auto group = [&](int s, int slot, auto uc, auto gc) {
        constexpr int U = decltype(uc)::value, g = decltype(gc)::value, H = g / MF, i = g % MF, ahead = g + kLead, d = U % 2, a = U % kSlots, next_a = (U + 1) % kSlots;
        constexpr bool first = ahead == kGroups;       // the first group whose reads ahead are the next step's
        constexpr int kFetch = MF == 8 ? 2 : 0, kRead = MF == 8 ? 4 : 2;
        constexpr int kPer = kParts;
        if constexpr (first) {
            // what may still be on its way: loads begun behind the next step's rows, and in a group's third step none of the
            // next group's weights, which the fourth one reads (of scales, one load at least)
            constexpr int kLater = (kSlots - 2) * A::kLoads, kWeights = U == 3 ? 3 : U == 0 ? (kSlots > 2 ? 5 : 2) : U == 1 && kSlots > 2 ? 5 : 0;
            arrive<kLater + kWeights>();
            fetch_a(s + kSlots, a);
        }
        read_a(Const<ahead % kGroups>{}, ahead < kGroups ? at.a ^ (a * kA) : at.a ^ (next_a * kA));
        if constexpr ((U == 3 || U == 0) && g == kFetch) {
            // half of the weights two groups on, where this group's are read; the other half a step later
            in_order();
            if constexpr (U == 3) {
                fetch_q(s / 4 + 2, slot, Const<0>{});
                scales = scales_of.load(s / 4 + 2);
            } else {
                fetch_q(s / 4 + 1, 1 - slot, Const<1>{});
            }
            in_order();
        }
        if constexpr (U == 2 && g == kFetch) put_s(scales, 1 - slot);
        if constexpr (g == kRead) read_b(Const<1 - d>{}, Const<(U + 1) % 4>{}, U == 3 ? 1 - slot : slot);
        if constexpr (g == MF) scale_of(Const<1 - d>{});
        auto part = [&](auto ec) {
            constexpr int e = g % MF * kPer + decltype(ec)::value;     // of the half's 2 NF
            if constexpr (H == 0) expand(Const<d>{}, Const<1>{}, Const<e / 2>{}, Const<e % 2>{});
            else expand(Const<1 - d>{}, Const<0>{}, Const<e / 2>{}, Const<e % 2>{});
        };
        part(Const<0>{});
        if constexpr (kPer >= 2) part(Const<1>{});
#pragma unroll
        for (int j = 0; j < NF; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[H][j]), __builtin_bit_cast(bf16x8, fa[g % kRing]),
                                                                acc[i][j], 0, 0, 0);
        // the order of a group: what else it does among its matrix instructions
        constexpr int kReads = 1 + (g == kRead ? 2 * NF : 0), kStarts = first ? A::kLoads : (U == 3 || U == 0) && g == kFetch ? 3 : 0;
#pragma unroll
        for (int r = 0; r < NF; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, (kReads + NF - 1) / NF, 0);                          // LDS reads
            if constexpr (kStarts > 0) __builtin_amdgcn_sched_group_barrier(0x010, (kStarts + NF - 1) / NF, 0);  // loads from memory
            __builtin_amdgcn_sched_group_barrier(0x002, 2 * kPer + (g == MF ? 3 : 0), 0);                    // vector instructions
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                               // matrix instructions
        }
    };
    static_assert((MF == 4 || MF == 8) && (kParts == 1 || kParts == 2), "groups of a step");
    auto step = [&](int s, int slot, auto uc) {
        group(s, slot, uc, Const<0>{}), group(s, slot, uc, Const<1>{}), group(s, slot, uc, Const<2>{}), group(s, slot, uc, Const<3>{});
        group(s, slot, uc, Const<4>{}), group(s, slot, uc, Const<5>{}), group(s, slot, uc, Const<6>{}), group(s, slot, uc, Const<7>{});
        if constexpr (MF >= 8) {
            group(s, slot, uc, Const<8>{}), group(s, slot, uc, Const<9>{}), group(s, slot, uc, Const<10>{}), group(s, slot, uc, Const<11>{});
            group(s, slot, uc, Const<12>{}), group(s, slot, uc, Const<13>{}), group(s, slot, uc, Const<14>{}), group(s, slot, uc, Const<15>{});
        }
        at.remake();
    };
    if (steps > 0) {
        scales = scales_of.load(0);
        fetch_q(0, 0, Const<0>{});
        fetch_q(0, 0, Const<1>{});
#pragma unroll
        for (int i = 0; i < kSlots; ++i) fetch_a(i, i);
        put_s(scales, 0);
        arrive<0>();
        fetch_q(1, 1, Const<0>{});
        scales = scales_of.load(1);
        in_order();
        read_b(Const<0>{}, Const<0>{}, 0);
        scale_of(Const<0>{});
        auto whole = [&](auto jc) { expand(Const<0>{}, Const<0>{}, jc, Const<0>{}), expand(Const<0>{}, Const<0>{}, jc, Const<1>{}); };
        whole(Const<0>{}), whole(Const<1>{});
        if constexpr (NF > 2) whole(Const<2>{}), whole(Const<3>{});
        read_a(Const<0>{}, at.a), read_a(Const<1>{}, at.a);
        if constexpr (kLead > 2) read_a(Const<2>{}, at.a);
        int slot = 0;
        for (int s = 0; s < steps; s += 4, slot = 1 - slot) {
            step(s, slot, Const<0>{});
            if (s + 1 < steps) step(s + 1, slot, Const<1>{});
            if (s + 2 < steps) step(s + 2, slot, Const<2>{});
            if (s + 3 < steps) step(s + 3, slot, Const<3>{});
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load into LDS outlives the workgroup
    finish<T, MF, NF>(p, t, n0, lds, tid, acc);
}

// The product of one tile with turned weights.
template <class T, int MF>
__device__ __forceinline__ void product_turned(const Args& p, const Place& t, int64_t n0, char* lds, int tid) {
    constexpr int NF = 4, kRows = MF * 32;
    using A = Side<kRows, T::kThreads, false>;
    using B = Turned<T>;
    const int lane = tid % kLanes, wave = __builtin_amdgcn_readfirstlane(tid / kLanes), wm = wave / T::WN, wn = wave % T::WN;
    A sa;
    sa.init(t.left, p.ld, tid);
    const char* a0 = p.x + t.first * p.ld;
    const int64_t row_bytes = p.inner * 2, q_ld = p.k / 2, s_ld = p.k >> p.shift;
    auto fetch_a = [&](int s, int slot) {
        sa.load(a0 + (int64_t)s * kStepBytes, nullptr, lds + slot * T::kStage, row_bytes - (int64_t)s * kStepBytes, tid, wave);
    };
    typename B::From at;
    at.init(p, n0, tid);
    const char* q0 = p.q + t.expert * p.n * q_ld + n0 / 2;
    const uint8_t* s0 = p.scales + t.expert * p.n * s_ld;
    const int64_t q_left = p.n * q_ld - n0 / 2, s_left = p.n * s_ld;
    auto fetch_b = [&](int s, B& b) {                      // the windows move down 64 rows a step
        const int64_t dq = s * 64 * q_ld, ds = s * 64 * s_ld;
        b.load(at, window_of(q0 + dq, q_left - dq), window_of(s0 + ds, s_left - ds));
    };
    auto a_row = [&](int i) { return wm * (MF * 16) + i * 16; };
    auto b_row = [&](int j) { return wn * 64 + j * 16; };
    f32x4 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // A step is 2 MF groups of NF matrix instructions, a fragment of the rows against a half's fragments of the weights.
    // Registers run kLead groups ahead of them (a whole half for the weights).  While a group is multiplied a later one's
    // fragment is read, and in the first groups the next step's weights are expanded and written, a part at a time; then
    // those of the step two behind it are loaded.  The one barrier of a step stands where its last fragments have been
    // read: behind it lie the next step's rows and weights, and its own LDS is free.
    constexpr int kLead = MF >= 8 ? 3 : MF >= 4 ? 2 : 1, kRing = 4, kGroups = 2 * MF;
    constexpr int kFetch = MF >= 8 ? 9 : MF;               // the group that loads weights
    const int steps = (int)((p.inner + 63) / 64);
    // Where this lane reads its chunk of a fragment's first half, and where it writes: chunks' places are exchanged by
    // their row, so other chunks and the next step's LDS are some bits away.  Made in each step, not kept for all.
    const int l16 = lane % 16, chunk = lane / 16;
    uint32_t a_at = (a_row(0) + l16) * kStepBytes + (chunk ^ A::exchange(l16)) * kChunk;
    uint32_t b_at = (T::M + b_row(0) + l16) * kStepBytes + (chunk ^ exchange(b_row(0) + l16)) * kChunk;
    uint32_t w_at = (uint32_t)(uintptr_t)(lds_void*)lds + T::M * kStepBytes + B::base(tid);   // the kernel's LDS begins with it
    static_assert((T::kStage & (T::kStage - 1)) == 0 && T::M * kStepBytes >= 1024, "bits apart");
    B b[2];
    i32x4 fa[kRing], fb[2][NF];
    auto read_a = [&](auto gc, uint32_t from) {            // the fragment of group g of a step
        constexpr int g = decltype(gc)::value;
        fa[g % kRing] = *reinterpret_cast<const i32x4*>(lds + (from ^ (g / MF * 64)) + g % MF * (16 * kStepBytes));
    };
    auto read_b = [&](auto hc, uint32_t stage, int from, int to) {
        constexpr int H = decltype(hc)::value;
#pragma unroll
        for (int j = from; j < to; ++j)
            fb[H][j] = *reinterpret_cast<const i32x4*>(lds + (stage ^ ((4 * H) ^ j) * kChunk) + j * (16 * kStepBytes));
    };
    auto in_order = [] { asm volatile("" ::: "memory"); };   // the waits count on it
    auto group = [&](int s, auto dc, auto gc) {
        constexpr int d = decltype(dc)::value, g = decltype(gc)::value, H = g / MF, i = g % MF, ahead = g + kLead;
        constexpr bool first = ahead == kGroups;       // the first group whose reads ahead are the next step's
        constexpr bool more_b = g < NF && g < MF - 1;  // the second half's weights: one in each of the first groups
        constexpr int b_to = g == MF - 2 ? NF : g + 1;
        constexpr int kReads = 1 + (more_b ? b_to - g : 0) + (first ? NF : 0);
        constexpr int kPer = MF == 2 ? 2 : 1;          // parts of the next step's weights
        constexpr bool stores = MF == 8 ? g % 2 == 1 && g < 8 : g * kPer < B::kParts;
        constexpr int part = MF == 8 ? g / 2 : g * kPer;
        if constexpr (first) {
            arrive<B::kLoads>();                       // the weights' loads go on
            fetch_a(s + 2, d);
            read_b(Const<0>{}, b_at ^ T::kStage, 0, NF);
        }
        read_a(Const<ahead % kGroups>{}, ahead < kGroups ? a_at : a_at ^ T::kStage);
        if constexpr (more_b) read_b(Const<1>{}, b_at, g, b_to);
        if constexpr (stores) {
            const uint32_t to = w_at ^ T::kStage;
            b[1 - d].template store<part>(to);
            if constexpr (kPer == 2) b[1 - d].template store<part + 1>(to);
        }
        if constexpr (g == kFetch) {
            in_order();
            fetch_b(s + 3, b[1 - d]);
        }
#pragma unroll
        for (int j = 0; j < NF; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[H][j]), __builtin_bit_cast(bf16x8, fa[g % kRing]),
                                                                acc[i][j], 0, 0, 0);
        // the order of a group: what else it does among its matrix instructions
#pragma unroll
        for (int r = 0; r < NF; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, (kReads + NF - 1) / NF, 0);                          // LDS reads
            if constexpr (first) __builtin_amdgcn_sched_group_barrier(0x010, (A::kLoads + NF - 1) / NF, 0);  // loads from memory
            if constexpr (g == kFetch) __builtin_amdgcn_sched_group_barrier(0x010, (B::kLoads + NF - 1) / NF, 0);
            if constexpr (stores) __builtin_amdgcn_sched_group_barrier(0x002, 5 * kPer, 0);                  // vector instructions
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                               // matrix instructions
        }
        if constexpr (g % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // not over all of a step: registers
    };
    static_assert(MF == 2 || MF == 4 || MF == 8, "groups of a step");
    auto step = [&](int s, auto dc) {
        group(s, dc, Const<0>{}), group(s, dc, Const<1>{}), group(s, dc, Const<2>{}), group(s, dc, Const<3>{});
        if constexpr (MF >= 4) group(s, dc, Const<4>{}), group(s, dc, Const<5>{}), group(s, dc, Const<6>{}), group(s, dc, Const<7>{});
        if constexpr (MF >= 8) {
            group(s, dc, Const<8>{}), group(s, dc, Const<9>{}), group(s, dc, Const<10>{}), group(s, dc, Const<11>{});
            group(s, dc, Const<12>{}), group(s, dc, Const<13>{}), group(s, dc, Const<14>{}), group(s, dc, Const<15>{});
        }
        a_at ^= T::kStage, b_at ^= T::kStage, w_at ^= T::kStage;
        asm volatile("" : "+v"(a_at), "+v"(b_at), "+v"(w_at));
        at.remake();
    };
    if (steps > 0) {
        fetch_b(0, b[0]);
        fetch_b(1, b[1]);
        in_order();
        fetch_a(0, 0);
        in_order();
        fetch_a(1, 1);
        in_order();
        b[0].template store<0>(w_at), b[0].template store<1>(w_at), b[0].template store<2>(w_at), b[0].template store<3>(w_at);
        fetch_b(2, b[0]);
        in_order();
        arrive<A::kLoads + B::kLoads>();
        read_b(Const<0>{}, b_at, 0, NF);
        read_a(Const<0>{}, a_at);
        if constexpr (kLead > 1) read_a(Const<1>{}, a_at);
        if constexpr (kLead > 2) read_a(Const<2>{}, a_at);
        for (int s = 0; s < steps; s += 2) {               // past the last step: zeros
            step(s, Const<0>{});
            step(s + 1, Const<1>{});
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no load into LDS outlives the workgroup
    finish<T, MF, NF>(p, t, n0, lds, tid, acc);
}

template <class T, bool TURNED>
__global__ __launch_bounds__(T::kThreads, 2) void grouped_kernel(Args p) {
    __shared__ __attribute__((aligned(1024))) char lds[TURNED ? kSteps * T::kStage : T::kLds];
    const int tid = threadIdx.x;
    const Offsets offsets = offsets_of(p, tid % kLanes);
    const Groups all = groups_of(p, offsets, T::M, tid % kLanes);
    const Work work = work_of<T::kSplit>(blockIdx.x, gridDim.x, all.tiles, p.tiles_n);
    if (!work.tile) return clear_rows(p, all, work, tid, T::kThreads);
    const int64_t n0 = work.n * T::N;
    Place t = place_of(p, offsets, work.index, T::M, tid % kLanes);
    if constexpr (T::kSplit) {
        const int64_t height = T::M / work.parts;
        t.first += work.part * height, t.left -= work.part * height;
        if (t.left <= 0) return;
        if (work.parts > 1 && t.left > height) t.left = height;
    }
    auto product = [&](auto mc) {
        constexpr int MF = decltype(mc)::value;            // 32 MF rows
        if constexpr (TURNED) product_turned<T, MF>(p, t, n0, lds, tid);
        // 64 rows: all of them and half as many weights a wave, which then expands half as many
        else if constexpr (MF == 2) product_raw<T, 4, 2>(p, t, n0, lds, tid);
        else product_raw<T, MF, 4>(p, t, n0, lds, tid);
    };
    if (t.left <= 64) return product(Const<2>{});
    if constexpr (T::kMost > 4) if (t.left <= 128) return product(Const<4>{});
    product(Const<T::kMost>{});
}

}  // namespace grouped_product
