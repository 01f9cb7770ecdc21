"""The products' operators in 64 bits on the CPU, from their formulas, and the bounds their kernels keep.

Bounds, elementwise: a sum of K products held in binary32 is off by at most (K + 2) 2^-24 sum |a b| in any
order; a rounding to bfloat16 (8 significand bits) adds 2^-8 |y|, one to binary32 2^-24 |y|."""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
SIGNED = torch.tensor(np.concatenate([GRID, -GRID]))
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SUM = 2.0 ** -24
# a binary32 logistic function of a binary32 argument: exponential, sum, reciprocal and the products around them,
# each off by a few 2^-23, the argument's own product by 2^-24 of at most 90 (e^-g is negligible beyond)
GATE = 2.0 ** -16


def f64(t):
    return t.detach().cpu().double()


def nibbles(q):
    q = q.cpu().long()
    return SIGNED[torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], q.shape[1] * 2)]


def e4m3(codes):
    return codes.cpu().contiguous().view(torch.float8_e4m3fn).double()


def nvfp4_values(q, scales, block):
    """q s, without the global scale."""
    v = nibbles(q)
    return v * e4m3(scales).reshape(v.shape[0], -1).repeat_interleave(block, 1)


def mx_values(q, scales):
    c = scales.cpu().double()
    s = torch.where(c == 255, torch.full_like(c, float("nan")), torch.exp2(c - 127))
    return nibbles(q) * s.repeat_interleave(32, 1)


def mx_quantize(x):
    """(values [rows, 32 kb], codes [rows, kb]) by nearest grid point, ties to the even code."""
    x = f64(x).numpy()
    rows, cols = x.shape
    kb = -(-cols // 32)
    y = np.zeros((rows, 32 * kb))
    y[:, :cols] = x
    y = y.reshape(rows, kb, 32)
    top = np.abs(y).max(-1) if kb else np.zeros((rows, 0))
    bad = ~np.isfinite(top)
    E = np.full(top.shape, -127.0)
    some = ~bad & (top > 0)
    E[some] = np.clip(np.floor(np.log2(top[some])) - 2, -127, 127)
    # floor(log2) from the exponent itself, not from a rounded logarithm
    E[some] = np.clip(np.frexp(top[some])[1] - 1 - 2, -127, 127)
    v = np.where(bad[..., None], 0.0, y) / np.exp2(E)[..., None]
    a = np.abs(v)
    d = np.abs(a[..., None] - GRID)
    low = d.argmin(-1)                                   # of two equally near ones the lower code
    up = np.minimum(low + 1, 7)
    tie = (np.take_along_axis(d, up[..., None], -1)[..., 0] == np.take_along_axis(d, low[..., None], -1)[..., 0]) & (low < 7)
    code = np.where(tie & (low % 2 == 1), up, low)
    val = np.copysign(GRID[code], v) * np.exp2(E)[..., None]
    val = np.where(bad[..., None], np.nan, val)
    codes = np.where(bad, 255, E + 127).astype(np.uint8)
    return torch.tensor(val.reshape(rows, 32 * kb)), torch.tensor(codes)


def product(a, b):
    """(a b^T, its bound without the output's rounding)."""
    k = a.shape[1]
    return a @ b.t(), (k + 2) * SUM * (a.abs() @ b.abs().t())


def silu(g):
    return g * torch.sigmoid(g)


def ffn(x, wg, wu):
    """h, g, u and their bounds without the outputs' rounding."""
    g, eg = product(f64(x), f64(wg))
    u, eu = product(f64(x), f64(wu))
    h = silu(g) * u
    # |silu'| < 1.1
    eh = (1.1 * eg * (u.abs() + eu) + (silu(g).abs() + 1.1 * eg) * eu) + GATE * h.abs()
    return (h, g, u), (eh, eg, eu)


def ffn_gates(dh, g, u):
    """dg, du and their bounds once rounded to bfloat16."""
    dh, g, u = f64(dh), f64(g), f64(u)
    s = torch.sigmoid(g)
    du = dh * g * s
    dg = dh * u * s * (1 + g * (1 - s))
    r = ROUND[torch.bfloat16]
    edu = (r + GATE) * du.abs()
    edg = r * dg.abs() + GATE * (dh * u).abs() * s * (1 + (g * (1 - s)).abs())
    return (dg, du), (edg, edu)


def ffn_grads(dh, x, wg, wu, g, u):
    """dx, dwg, dwu and their bounds without the outputs' rounding."""
    (dg, du), (edg, edu) = ffn_gates(dh, g, u)
    x, wg, wu = f64(x), f64(wg), f64(wu)
    m, n = dg.shape

    def both(d, e, w, k):
        return d @ w, e @ w.abs() + (k + 2) * SUM * ((d.abs() + e) @ w.abs())

    a, ea = both(dg, edg, wg, 2 * n)
    b, eb = both(du, edu, wu, 2 * n)
    c, ec = both(dg.t(), edg.t(), x, m)
    d, ed = both(du.t(), edu.t(), x, m)
    return (a + b, c, d), (ea + eb, ec, ed)


def check(got, want, bound, what=""):
    """got within its bound of want, after the rounding of its own type."""
    r = ROUND[got.dtype]
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    lim = bound + r * (want.abs() + bound) + 1e-40
    off = (g - want).abs()
    ok = (off <= lim) | (g.isnan() & want.isnan())
    assert bool(ok.all()), (what, f"{int((~ok).sum())} of {ok.numel()} off, worst "
                            f"{float((off / lim)[~ok].max()):.3g} times the bound at {(~ok).nonzero()[0].tolist()}")


def between_nans(t, pad_rows=8, pad_cols=24):
    """The same matrix as a 16-byte aligned view of a storage whose other values are NaN."""
    big = torch.full((t.shape[0] + 2 * pad_rows, t.shape[1] + pad_cols), float("nan"), dtype=t.dtype, device=t.device)
    view = big[pad_rows:pad_rows + t.shape[0], 8:8 + t.shape[1]]
    view.copy_(t)
    return view
