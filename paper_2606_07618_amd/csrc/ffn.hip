// Gated feed-forward block on AMD Instinct MI355X (gfx950): g = x Wg^T, u = x Wu^T,
// h = silu(g) u, silu(g) = g / (1 + e^-g), in bfloat16 with sums in binary32, and its backward pass
//   s = 1 / (1 + e^-g),  dg = dh u s (1 + g (1 - s)),  du = dh g s,
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.
#include "dot_product.h"
#include "product_host.h"
#include "thin_product.h"

namespace {

using namespace product_host;

constexpr int kEdgeThreads = 256;

__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// dg and du, side by side: d [m, ld], du from column `half` on, zeros from n to half.  Their rounding to
// bfloat16 is what the matrix cores take; the products' sums stay in binary32.
template <bool VEC>
__global__ __launch_bounds__(kEdgeThreads) void gate_grad_kernel(const uint16_t* __restrict__ dh,
                                                                 const uint16_t* __restrict__ gate,
                                                                 const uint16_t* __restrict__ up_, int64_t m, int64_t n,
                                                                 int64_t half, int64_t ld, uint16_t* __restrict__ d) {
    const int64_t row_units = half / 8, units = m * row_units;
    for (int64_t i = (int64_t)blockIdx.x * kEdgeThreads + threadIdx.x; i < units;
         i += (int64_t)gridDim.x * kEdgeThreads) {
        const int64_t r = i / row_units, c = i % row_units * 8;
        uint16_t a[8], g[8], u[8];
        if (VEC && c < n) {
            *reinterpret_cast<uint4*>(a) = *reinterpret_cast<const uint4*>(dh + r * n + c);
            *reinterpret_cast<uint4*>(g) = *reinterpret_cast<const uint4*>(gate + r * n + c);
            *reinterpret_cast<uint4*>(u) = *reinterpret_cast<const uint4*>(up_ + r * n + c);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = c + j < n;
                a[j] = in ? dh[r * n + c + j] : 0;
                g[j] = in ? gate[r * n + c + j] : 0;
                u[j] = in ? up_[r * n + c + j] : 0;
            }
        }
        uint32_t og[4], ou[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float dg[2], du[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float G = bf16_f32(g[2 * j + e]), U = bf16_f32(u[2 * j + e]), H = bf16_f32(a[2 * j + e]);
                const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(G * -1.44269504f));
                const float silu = G * s;
                du[e] = H * silu;
                dg[e] = H * U * fmaf(silu, 1.0f - s, s);
            }
            og[j] = pack_bf16(dg[0], dg[1]);
            ou[j] = pack_bf16(du[0], du[1]);
        }
        *reinterpret_cast<uint4*>(d + r * ld + c) = make_uint4(og[0], og[1], og[2], og[3]);
        *reinterpret_cast<uint4*>(d + r * ld + half + c) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
    }
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

int64_t pack_workspace(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    Carver c{nullptr};
    if (needs_pack(k, ldx)) c.take(m * packed_ld(k) * 2);
    if (needs_pack(k, ldw)) {
        c.take(n * packed_ld(k) * 2);
        c.take(n * packed_ld(k) * 2);
    }
    return c.at;
}

int64_t half_of(int64_t n) { return up(n, 64); }       // whole steps of the contraction

int64_t backward_workspace(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    return pack_workspace(m, n, k, ldx, ldw) + up(m * 2 * half_of(n) * 2, 256) + parts_bytes<kBf16, kAcross, kPairInner>(m, k, n);
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
    return pack_workspace(m, n, k, ldx, ldw);
}

int nvfp4_swiglu_ffn(const void* x, int64_t ldx, const void* w_gate, const void* w_up, int64_t ldw, int64_t m,
                     int64_t n, int64_t k, void* h, void* gate, void* up_out, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    if (m == 0 || n == 0) return NVFP4_OK;
    if (!h || (k > 0 && (!x || !w_gate || !w_up)) || !gate != !up_out) return NVFP4_ERR_NULL;
    if (!aligned(x, 16) || !aligned(w_gate, 16) || !aligned(w_up, 16) || !aligned(h, 16) || !aligned(gate, 16) ||
        !aligned(up_out, 16))
        return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, pack_workspace(m, n, k, ldx, ldw))) return rc;
    hipStream_t st = (hipStream_t)stream;
    Carver c{static_cast<char*>(workspace)};
    Rows rx{x, ldx}, rg{w_gate, ldw}, ru{w_up, ldw};
    const bool pw = needs_pack(k, ldw);
    if (const int rc = packed(c, rx, m, k, needs_pack(k, ldx), st)) return rc;
    if (const int rc = packed(c, rg, n, k, pw, st)) return rc;
    if (const int rc = packed(c, ru, n, k, pw, st)) return rc;
    if (m <= dot_product::kMostRows) {
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
    if (m <= thin_product::kRows) {
        thin_product::Args t = {};
        t.w = static_cast<const char*>(rg.p), t.w2 = static_cast<const char*>(ru.p), t.ldw = rg.ld * 2;
        t.x = static_cast<const char*>(rx.p), t.ldx = rx.ld * 2, t.m = (int)m, t.n = n, t.k = k;
        t.out = h, t.out2 = gate, t.out3 = up_out;
        thin_product::launch_thin<thin_product::kGated, 8, 4, true>(t, st);
        return launched();
    }
    Args p = {};
    p.a.p = static_cast<const char*>(rx.p), p.a.ld = rx.ld * 2;
    p.b.p = static_cast<const char*>(rg.p), p.b.p2 = static_cast<const char*>(ru.p), p.b.ld = rg.ld * 2;
    p.m = m, p.n = n, p.inner = k, p.out = h, p.out2 = gate, p.out3 = up_out, p.out_ld = n;
    p.parts = 1;
    return launch_product<kBf16, kAlong, kAlong, kPairOuter, kGate>(p, plan_product<kBf16, kAlong, kPairOuter>(m, n, k, false).tile, st);
}

int64_t nvfp4_swiglu_ffn_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    return backward_workspace(m, n, k, ldx, ldw);
}

int nvfp4_swiglu_ffn_backward(const void* dh, const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                              int64_t ldw, const void* gate, const void* up_in, int64_t m, int64_t n, int64_t k,
                              void* dx, void* dw_gate, void* dw_up, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (const int rc = check_call(m, n, k, ldx, ldw)) return rc;
    const bool inputs = m > 0 && n > 0;
    const bool want_x = dx && m > 0 && k > 0, want_w = dw_gate && n > 0 && k > 0;
    if (!dw_gate != !dw_up) return NVFP4_ERR_NULL;
    if (!dx && !dw_gate && m * n * k > 0) return NVFP4_ERR_NULL;
    if (!want_x && !want_w) return NVFP4_OK;
    if (inputs && (!dh || !gate || !up_in || (want_x && (!w_gate || !w_up)) || (want_w && !x))) return NVFP4_ERR_NULL;
    for (const void* p : {dh, x, w_gate, w_up, gate, up_in, (const void*)dx, (const void*)dw_gate, (const void*)dw_up})
        if (!aligned(p, 16)) return NVFP4_ERR_ALIGN;
    if (const int rc = check_ws(workspace, workspace_bytes, backward_workspace(m, n, k, ldx, ldw))) return rc;
    hipStream_t st = (hipStream_t)stream;
    Carver c{static_cast<char*>(workspace)};
    const int64_t half = half_of(n);
    const int64_t ld = 2 * half;
    uint16_t* d = static_cast<uint16_t*>(c.take(m * ld * 2));
    const int64_t units = m * (half / 8), groups = ceil_div(units, kEdgeThreads);
    if (units > 0) {
        hipLaunchKernelGGL((n % 8 == 0 ? gate_grad_kernel<true> : gate_grad_kernel<false>),
                           dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(kEdgeThreads), 0, st,
                           static_cast<const uint16_t*>(dh), static_cast<const uint16_t*>(gate),
                           static_cast<const uint16_t*>(up_in), m, n, half, ld, d);
        if (const int rc = launched()) return rc;
    }
    Rows rx{x, ldx}, rg{w_gate, ldw}, ru{w_up, ldw};
    if (want_x) {
        const bool pw = needs_pack(k, ldw);
        if (const int rc = packed(c, rg, n, k, pw, st)) return rc;
        if (const int rc = packed(c, ru, n, k, pw, st)) return rc;
        Args p = {};
        p.a.p = reinterpret_cast<const char*>(d), p.a.ld = ld * 2;
        p.b.p = static_cast<const char*>(rg.p), p.b.p2 = static_cast<const char*>(ru.p), p.b.ld = rg.ld * 2;
        p.m = m, p.n = k, p.inner = n, p.out = dx, p.out_ld = k;
        if (const int rc = run_sums<kBf16, kAlong, kAcross, kPairInner>(p, static_cast<float*>(c.take(0)), st)) return rc;
    }
    if (want_w) {
        if (const int rc = packed(c, rx, m, k, needs_pack(k, ldx), st)) return rc;
        Args p = {};
        p.a.p = reinterpret_cast<const char*>(d), p.a.ld = ld * 2;
        p.b.p = static_cast<const char*>(rx.p), p.b.ld = rx.ld * 2;
        p.m = 2 * half, p.n = k, p.inner = m, p.half_rows = half, p.out_rows = n;
        p.out = dw_gate, p.out2 = dw_up, p.out_ld = k;
        p.parts = 1;
        const int tile = plan_product<kBf16, kAcross, kSingle>(p.m, k, m, false).tile;
        if (const int rc = launch_product<kBf16, kAcross, kAcross, kSingle, kTwoRows>(p, tile, st)) return rc;
    }
    return NVFP4_OK;
}

}  // extern "C"
