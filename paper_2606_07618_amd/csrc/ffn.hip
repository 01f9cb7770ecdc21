// Gated feed-forward block on AMD Instinct MI355X (gfx950): g = x Wg^T, u = x Wu^T,
// h = silu(g) u, silu(g) = g / (1 + e^-g), in bfloat16 with sums in binary32, and its backward pass
//   s = 1 / (1 + e^-g),  dg = dh u s (1 + g (1 - s)),  du = dh g s,
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.
#include "dot_product.h"
#include "product_host.h"

namespace {

using namespace product_host;

constexpr int kEdgeThreads = 256;

// The backward products' contractions run over the tokens (dW) and over the weights' rows (dx), so dg and du are
// written as they lie and turned, and x and the weights are turned: all four products then read whole rows.  One launch
// does all of it (prepare_kernel): with six launches a gradient of [237, 176] -> 112 took 31 us, with three 22.
// [4000, 4096] -> 14336: 1830 us with the operands as they lie, 1636 so.  The two products take 1.39 to 1.43 ms of it
// (1.31 to 1.35 PFLOP/s), the preparation 244 us for the 1.34 GB it has to move (5.5 TB/s).
//
// Turning: a workgroup takes 64 rows by 128 columns.  A thread holds two rows by eight columns of either half and
// writes pairs of rows, a word each, to LDS; LDS rows are a word longer than their 64 values, so that the eight row
// pairs by eight groups of columns of a wave meet in no bank.  Then each row of LDS leaves in 16-byte pieces.
constexpr int kTurnRows = 64, kTurnColumns = 128;
typedef uint32_t TurnTile[kTurnColumns][kTurnRows / 2 + 1];

constexpr int kTurnHalf = kTurnColumns / 2;
__device__ __forceinline__ int turn_pair() { return threadIdx.x / 8; }
__device__ __forceinline__ int turn_column() { return threadIdx.x % 8 * 8; }

// Words of two rows' eight values to columns c .. c + 7.
__device__ __forceinline__ void turn8(TurnTile& tile, int c, const uint4& a, const uint4& b) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        tile[c + 2 * j][turn_pair()] = __builtin_amdgcn_perm(y[j], x[j], 0x05040100u);
        tile[c + 2 * j + 1][turn_pair()] = __builtin_amdgcn_perm(y[j], x[j], 0x07060302u);
    }
}

// Columns c0 .. of the source as rows of dst, values r0 .. r0 + 63 of each, as far as they lie in [rows, fill].
__device__ __forceinline__ void turn_out(const TurnTile& tile, int64_t c0, int64_t rows, int64_t r0, int64_t fill,
                                         int64_t to_ld, uint16_t* dst) {
#pragma unroll
    for (int i = 0; i < kTurnColumns * kTurnRows / 8 / kEdgeThreads; ++i) {
        const int at = i * kEdgeThreads + threadIdx.x, c = at / (kTurnRows / 8), chunk = at % (kTurnRows / 8);
        if (c0 + c < rows && r0 + chunk * 8 < fill)
            *reinterpret_cast<uint4*>(dst + (c0 + c) * to_ld + r0 + chunk * 8) =
                make_uint4(tile[c][chunk * 4], tile[c][chunk * 4 + 1], tile[c][chunk * 4 + 2], tile[c][chunk * 4 + 3]);
    }
}

// Values c .. c + 7 of row r of a [rows, width] matrix, zeros outside.  vec: its rows are whole 16-byte pieces.
__device__ __forceinline__ uint4 eight(bool vec, const uint16_t* src, int64_t r, int64_t rows, int64_t c, int64_t width,
                                       int64_t ld) {
    if (r >= rows || c >= width) return make_uint4(0, 0, 0, 0);
    if (vec) return *reinterpret_cast<const uint4*>(src + r * ld + c);
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < width ? src[r * ld + c + j] : 0u;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// src [rows, width] turned: dst [width, to_ld], values from rows to fill zero.  vec: rows are whole 16-byte pieces.
struct Turn { const uint16_t* src; int64_t rows, width, ld, fill; uint16_t* dst; int64_t to_ld; uint32_t tiles_c, tiles; int vec; };

__device__ __forceinline__ void turn(TurnTile& tile, const Turn& p, uint32_t at) {
    const int64_t r0 = (int64_t)(at / p.tiles_c) * kTurnRows, c0 = (int64_t)(at % p.tiles_c) * kTurnColumns;
    const int64_t r = r0 + turn_pair() * 2, c = c0 + turn_column();
    uint4 v[2][2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            v[h][e] = eight(p.vec, p.src, r + e, p.rows, c + h * kTurnHalf, p.width, p.ld);
#pragma unroll
    for (int h = 0; h < 2; ++h) turn8(tile, turn_column() + h * kTurnHalf, v[h][0], v[h][1]);
    __syncthreads();
    turn_out(tile, c0, p.width, r0, p.fill, p.to_ld, p.dst);
}

// dg and du side by side, d [m, 2 half], du from column `half` on, zeros from n to half; and turned, one below the
// other, t [2 n, ld], zeros from m to ld.  Either is left out where its pointer is NULL.  Their rounding to
// bfloat16 is what the matrix cores take; the products' sums stay in binary32.  It takes the gradients' error, relative
// and in the mean square, from 0.0017 (that of their own rounding) to 0.0024; dg and du as two bfloat16 numbers each
// would take it back and twice the matrix work.
struct Gates { const uint16_t *dh, *gate, *up; int64_t m, n, half; uint16_t* d; int64_t ld; uint16_t* t; uint32_t tiles_n, tiles; };

__device__ __forceinline__ void gate_grad(TurnTile& tg, TurnTile& tu, const Gates& p, uint32_t at) {
    const int64_t m = p.m, n = p.n, half = p.half, ld = p.ld;
    uint16_t *d = p.d, *t = p.t;
    const bool vec = n % 8 == 0;
    const int64_t r0 = (int64_t)(at / p.tiles_n) * kTurnRows, c0 = (int64_t)(at % p.tiles_n) * kTurnColumns;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t r = r0 + turn_pair() * 2, c = c0 + turn_column() + h * kTurnHalf;
        uint4 og[2], ou[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint4 va = eight(vec, p.dh, r + e, m, c, n, n), vg = eight(vec, p.gate, r + e, m, c, n, n),
                        vu = eight(vec, p.up, r + e, m, c, n, n);
            const uint32_t a[4] = {va.x, va.y, va.z, va.w}, g[4] = {vg.x, vg.y, vg.z, vg.w}, u[4] = {vu.x, vu.y, vu.z, vu.w};
            uint32_t wg[4], wu[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float dg[2], du[2];
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int shift = o ? 0 : 16;
                    const float G = __uint_as_float(g[j] << shift & 0xFFFF0000u), U = __uint_as_float(u[j] << shift & 0xFFFF0000u),
                                H = __uint_as_float(a[j] << shift & 0xFFFF0000u);
                    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(G * -1.44269504f));
                    const float silu = G * s;
                    du[o] = H * silu;
                    dg[o] = H * U * fmaf(silu, 1.0f - s, s);
                }
                wg[j] = pack_bf16(dg[0], dg[1]);
                wu[j] = pack_bf16(du[0], du[1]);
            }
            og[e] = make_uint4(wg[0], wg[1], wg[2], wg[3]);
            ou[e] = make_uint4(wu[0], wu[1], wu[2], wu[3]);
            if (d && r + e < m && c < half) {
                *reinterpret_cast<uint4*>(d + (r + e) * 2 * half + c) = og[e];
                *reinterpret_cast<uint4*>(d + (r + e) * 2 * half + half + c) = ou[e];
            }
        }
        if (t) {
            turn8(tg, turn_column() + h * kTurnHalf, og[0], og[1]);
            turn8(tu, turn_column() + h * kTurnHalf, ou[0], ou[1]);
        }
    }
    if (!t) return;
    __syncthreads();
    turn_out(tg, c0, n, r0, ld, ld, t);
    turn_out(tu, c0, n, r0, ld, ld, t + n * ld);
}

// Everything that the products wait for, in one launch: workgroups of dg and du first, then those of the turned operands.
struct Prepare { Gates gates; Turn turns[3]; };

__global__ __launch_bounds__(kEdgeThreads) void prepare_kernel(Prepare p) {
    __shared__ TurnTile tile[2];
    uint32_t at = blockIdx.x;
    if (at < p.gates.tiles) return gate_grad(tile[0], tile[1], p.gates, at);
    at -= p.gates.tiles;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (at < p.turns[i].tiles) return turn(tile[0], p.turns[i], at);
        at -= p.turns[i].tiles;
    }
}

int64_t turn_tiles(int64_t rows, int64_t columns) { return ceil_div(rows, kTurnRows) * ceil_div(columns, kTurnColumns); }

// The tiles of p, all of them; a launch takes most_groups(kEdgeThreads) of them.
int64_t count_tiles(Prepare& p) {
    int64_t tiles = 0;
    const auto count = [&](int64_t rows, int64_t columns, uint32_t& across, uint32_t& all) {
        across = (uint32_t)ceil_div(columns, kTurnColumns), all = (uint32_t)turn_tiles(rows, columns);
        tiles += turn_tiles(rows, columns);
    };
    count(p.gates.m, p.gates.n, p.gates.tiles_n, p.gates.tiles);
    for (Turn& t : p.turns) {
        t.vec = t.width % 8 == 0 && t.ld % 8 == 0;
        count(t.fill, t.width, t.tiles_c, t.tiles);
    }
    return tiles;
}

int prepare(Prepare& p, hipStream_t stream) {
    const int64_t tiles = count_tiles(p);
    if (tiles == 0) return NVFP4_OK;
    if (!launchable(tiles, kEdgeThreads)) return NVFP4_ERR_SHAPE;
    hipLaunchKernelGGL(prepare_kernel, dim3((unsigned)tiles), dim3(kEdgeThreads), 0, stream, p);
    return launched();
}

struct Rows { const void* p; int64_t ld; };

// x and the weights as the tiles read them; the copies, where needed, lie in the workspace.
int packed(Carver& c, Rows& r, int64_t rows, int64_t width, bool pack, hipStream_t stream) {
    if (!pack) return NVFP4_OK;
    void* to = c.take(rows * packed_ld(width) * 2);
    if (const int rc = pack_bf16_rows(r.p, rows, width, r.ld, to, stream)) return rc;
    r = {to, packed_ld(width)};
    return NVFP4_OK;
}

// h, and both pre-activations where asked for, from the sums of parts of the contraction, added in order.
template <bool VEC>
__global__ __launch_bounds__(kEdgeThreads) void join_gate_kernel(const float* __restrict__ part, int parts, int64_t count,
                                                                 void* __restrict__ h, void* __restrict__ gate,
                                                                 void* __restrict__ up_) {
    constexpr int kPer = VEC ? 4 : 1;
    const int64_t at = ((int64_t)blockIdx.x * kEdgeThreads + threadIdx.x) * kPer;
    if (at >= count) return;
    f32x4 v[2] = {};
    for (int p = 0; p < parts; ++p)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float* from = part + (p * 2 + b) * count + at;
            if constexpr (VEC) v[b] += *reinterpret_cast<const f32x4*>(from);
            else v[b][0] += *from;
        }
    f32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = silu(v[0][e]) * v[1][e];
    store4(h, 0, at, kPer, VEC, out);
    if (gate) {
        store4(gate, 0, at, kPer, VEC, v[0]);
        store4(up_, 0, at, kPer, VEC, v[1]);
    }
}

int64_t forward_workspace(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    Carver c{nullptr};
    if (needs_pack(k, ldx)) c.take(m * packed_ld(k) * 2);
    if (needs_pack(k, ldw)) {
        c.take(n * packed_ld(k) * 2);
        c.take(n * packed_ld(k) * 2);
    }
    return c.at + (m > kDotRows ? parts_bytes<kBf16, kGate>(m, n, k) : 0);
}

// Sections of the backward pass's workspace, of the gradients asked for: d and the turned weights for dx, the turned d
// and x for the weights' gradients.
struct Backward { int64_t half, ld; char *d, *wt, *dt, *xt, *parts; };

int64_t backward_sections(void* workspace, int64_t m, int64_t n, int64_t k, bool want_x, bool want_w, Backward& b) {
    Carver c{static_cast<char*>(workspace)};
    // Whole lines of memory, and whole steps of the products: dW of [4000, 4096] -> 14336 took 842 us with rows
    // filled up to eights only, 770 so.
    b.half = up(n, 64), b.ld = up(m, 64);
    const auto take = [&](bool want, int64_t bytes) { return want ? static_cast<char*>(c.take(bytes)) : nullptr; };
    b.d = take(want_x, m * 2 * b.half * 2);
    b.dt = take(want_w, 2 * n * b.ld * 2);
    b.wt = take(want_x, k * 2 * b.half * 2);
    b.xt = take(want_w, k * b.ld * 2);
    const int64_t px = want_x ? parts_bytes<kBf16>(m, k, 2 * b.half) : 0,
                  pw = want_w ? parts_bytes<kBf16, kTwoRows>(2 * n, k, m) : 0;
    b.parts = static_cast<char*>(c.take(px > pw ? px : pw));     // of one product after the other
    return c.at;
}

bool forward_launchable(int64_t m, int64_t n, int64_t k) {
    return m <= kDotRows || product_launchable<kBf16, kGate>(m, n, k);
}

bool backward_launchable(int64_t m, int64_t n, int64_t k, bool want_x, bool want_w) {
    const int64_t half = up(n, 64);
    const int64_t tiles = turn_tiles(m, n) + (want_x ? 2 * turn_tiles(half, k) : 0) + (want_w ? turn_tiles(up(m, 64), k) : 0);
    return launchable(tiles, kEdgeThreads) && (!want_x || product_launchable<kBf16>(m, k, 2 * half)) &&
           (!want_w || product_launchable<kBf16, kTwoRows>(2 * n, k, m));
}

int check_call(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    if (const int rc = check_dims(m, n, k)) return rc;
    if (ldx < k || ldw < k || ldx > kMaxLd || ldw > kMaxLd) return NVFP4_ERR_SHAPE;
    return NVFP4_OK;
}

int check_ws(const void* ws, size_t bytes, int64_t need) {
    if (need > 0 && (!ws || (int64_t)bytes < need)) return NVFP4_ERR_WORKSPACE;
    return aligned(ws, 256) || need == 0 ? NVFP4_OK : NVFP4_ERR_ALIGN;
}

}  // namespace

extern "C" {

int64_t nvfp4_swiglu_ffn_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    return forward_workspace(m, n, k, ldx, ldw);
}

int nvfp4_swiglu_ffn(const void* x, int64_t ldx, const void* w_gate, const void* w_up, int64_t ldw, int64_t m,
                     int64_t n, int64_t k, void* h, void* gate, void* up_out, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    if (!forward_launchable(m, n, k)) return NVFP4_ERR_SHAPE;
    if (m == 0 || n == 0) return NVFP4_OK;
    if (!h || (k > 0 && (!x || !w_gate || !w_up)) || !gate != !up_out) return NVFP4_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w_gate, 16) || !aligned(w_up, 16) || !aligned(h, 16) || !aligned(gate, 16) ||
        !aligned(up_out, 16))
        return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, forward_workspace(m, n, k, ldx, ldw))) return rc;
    hipStream_t st = (hipStream_t)stream;
    Carver c{static_cast<char*>(workspace)};
    Rows rx{x, ldx}, rg{w_gate, ldw}, ru{w_up, ldw};
    const bool pw = needs_pack(k, ldw);
    if (const int rc = packed(c, rx, m, k, needs_pack(k, ldx), st)) return rc;
    if (const int rc = packed(c, rg, n, k, pw, st)) return rc;
    if (const int rc = packed(c, ru, n, k, pw, st)) return rc;
    if (m <= kDotRows) {
        dot_product::GatedArgs t = {};
        t.wg = static_cast<const char*>(rg.p), t.wu = static_cast<const char*>(ru.p), t.ldw = rg.ld * 2;
        t.x = static_cast<const char*>(rx.p), t.ldx = rx.ld * 2, t.n = n, t.k = k;
        t.along = dot_product::waves_along(k, dot_product::kGatedSpan);
        t.h = h, t.gate = gate, t.up = up_out;
        switch (m) {
            case 1: dot_product::launch_gated_dot<1>(t, st); break;
            case 2: dot_product::launch_gated_dot<2>(t, st); break;
            case 3: dot_product::launch_gated_dot<3>(t, st); break;
            default: dot_product::launch_gated_dot<4>(t, st);
        }
        return launched();
    }
    Args p = {};
    p.a.p = static_cast<const char*>(rx.p), p.a.ld = rx.ld * 2;
    p.b.p = static_cast<const char*>(rg.p), p.b.p2 = static_cast<const char*>(ru.p), p.b.ld = rg.ld * 2;
    p.m = m, p.n = n, p.inner = k, p.out = h, p.out2 = gate, p.out3 = up_out, p.out_ld = n;
    const Plan plan = plan_product<kBf16, kGate>(m, n, k);
    p.parts = plan.parts;
    if (plan.parts == 1) return launch_product<kBf16, kGate>(p, plan.tile, st);
    float* parts = static_cast<float*>(p.out = c.take(0));
    if (const int rc = launch_product<kBf16, kGatePartial>(p, plan.tile, st)) return rc;
    const bool vec = n % 4 == 0;
    const int64_t groups = ceil_div(vec ? m * n / 4 : m * n, kEdgeThreads);
    if (!launchable(groups, kEdgeThreads)) return NVFP4_ERR_SHAPE;
    hipLaunchKernelGGL((vec ? join_gate_kernel<true> : join_gate_kernel<false>), dim3((unsigned)groups), dim3(kEdgeThreads), 0, st,
                       parts, plan.parts, m * n, h, gate, up_out);
    return launched();
}

int64_t nvfp4_swiglu_ffn_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    return nvfp4_ffn_gradients_workspace_bytes(m, n, k, ldx, ldw, 1, 1);
}

int64_t nvfp4_ffn_gradients_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw, int want_x,
                                            int want_w) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    Backward b;
    return backward_sections(nullptr, m, n, k, want_x != 0, want_w != 0, b);
}

int nvfp4_swiglu_ffn_backward(const void* dh, const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                              int64_t ldw, const void* gate, const void* up_in, int64_t m, int64_t n, int64_t k,
                              void* dx, void* dw_gate, void* dw_up, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    const bool inputs = m > 0 && n > 0;
    const bool want_x = dx && m > 0 && k > 0, want_w = dw_gate && n > 0 && k > 0;
    if (!dw_gate != !dw_up) return NVFP4_ERR_NULL;
    if (!dx && !dw_gate && m > 0 && n > 0 && k > 0) return NVFP4_ERR_NULL;
    if (!want_x && !want_w) return NVFP4_OK;
    if (!backward_launchable(m, n, k, want_x, want_w)) return NVFP4_ERR_SHAPE;
    if (inputs && (!dh || !gate || !up_in || (want_x && (!w_gate || !w_up)) || (want_w && !x))) return NVFP4_ERR_NULL;
    for (const void* p : {dh, x, w_gate, w_up, gate, up_in, (const void*)dx, (const void*)dw_gate, (const void*)dw_up})
        if (!aligned(p, 16)) return NVFP4_ERR_ALIGN;
    if (want_w && m > kMaxLd) return NVFP4_ERR_SHAPE;              // a row of the turned operands
    Backward b;
    if (const int rc = check_ws(workspace, workspace_bytes, backward_sections(workspace, m, n, k, want_x, want_w, b))) return rc;
    hipStream_t st = (hipStream_t)stream;
    const auto values = [](const void* p) { return static_cast<const uint16_t*>(p); };
    const auto turned = [](char* p) { return reinterpret_cast<uint16_t*>(p); };
    Prepare ready = {};
    ready.gates = {values(dh), values(gate), values(up_in), m, n, b.half, want_x ? turned(b.d) : nullptr, b.ld,
                   want_w ? turned(b.dt) : nullptr};
    if (want_x) {
        ready.turns[0] = {values(w_gate), n, k, ldw, b.half, turned(b.wt), 2 * b.half};
        ready.turns[1] = {values(w_up), n, k, ldw, b.half, turned(b.wt) + b.half, 2 * b.half};
    }
    if (want_w) ready.turns[2] = {values(x), m, k, ldx, b.ld, turned(b.xt), b.ld};
    if (const int rc = prepare(ready, st)) return rc;
    if (want_x) {
        Args p = {};
        p.a.p = b.d, p.a.ld = p.b.ld = 2 * b.half * 2, p.b.p = b.wt;
        p.m = m, p.n = k, p.inner = 2 * b.half, p.out = dx, p.out_ld = k;
        if (const int rc = run_sums<kBf16>(p, reinterpret_cast<float*>(b.parts), st)) return rc;
    }
    if (want_w) {
        Args p = {};
        p.a.p = b.dt, p.a.ld = p.b.ld = b.ld * 2, p.b.p = b.xt;
        p.m = 2 * n, p.n = k, p.inner = m, p.half_rows = n;
        p.out = dw_gate, p.out2 = dw_up, p.out_ld = k;
        if (const int rc = run_sums<kBf16, kTwoRows>(p, reinterpret_cast<float*>(b.parts), st)) return rc;
    }
    return NVFP4_OK;
}

}  // extern "C"
