"""The products that follow quantization and the gated feed-forward block, as cases that can be
timed and compared.

``run`` computes a case either in elementary torch operations in 32 bits (``own`` false) or through
the package's entry points (``own`` true).  The kinds:

  mx_round_trip  microscaled FP4 of an activation or weight (E8M0 scale for each 32 values of a
                 row), and back: simulated quantization
  mx_linear      a linear layer on microscaled FP4 weights: the activation is quantized, then
                 multiplied with them
  linear         a linear layer on NVFP4 weights, activation in bfloat16
  linear_grad    its gradient with respect to the activation, for adapters trained through frozen
                 4-bit weights (NVFP4 or microscaled)
  ffn            h = silu(x Wg^T) (x Wu^T), with the pre-activations kept where a backward follows
  ffn_grad       its gradients with respect to x, Wg and Wu
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# Midpoints of neighbouring E2M1 values; a tie goes to the even code, so up at every second one.
MIDPOINTS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))
MOST_FLOPS = 1_900_000_000_000    # of a drawn case: the listed gated block
MOST_ELEMENTS = 117_440_512       # of a drawn round trip: 8192 rows of width 14336


def listed():
    return [
        # Eight tokens of a decode step ahead of a projection of a hidden-4096 model: launches and latency.
        {"name": "mx_round_trip_tokens", "kind": "mx_round_trip", "rows": 8, "cols": 4096, "dtype": "bf16"},
        # The input of the down projection for 8192 tokens of an 8B model, quantized in simulation.
        {"name": "mx_round_trip_mlp", "kind": "mx_round_trip", "rows": 8192, "cols": 14336, "dtype": "bf16"},
        # One token of one sequence through a gate projection: reading the weights is all there is.
        {"name": "mx_linear_token", "kind": "mx_linear", "rows": 1, "out": 14336, "in": 4096,
         "dtype": "bf16", "out_dtype": "bf16"},
        # A prompt of 777 tokens through a down projection cut for a shard of 1001 output channels, sums
        # kept in binary32 for a later reduction over shards: ragged in both directions.
        {"name": "mx_linear_ragged", "kind": "mx_linear", "rows": 777, "out": 1001, "in": 14336,
         "dtype": "f32", "out_dtype": "f32"},
        # A prompt of 8192 tokens through the gate projection of an 8B model.
        {"name": "mx_linear_prompt", "kind": "mx_linear", "rows": 8192, "out": 14336, "in": 4096,
         "dtype": "bf16", "out_dtype": "bf16"},
        # One token through the down projection of an 8B model.
        {"name": "linear_token", "kind": "linear", "rows": 1, "out": 4096, "in": 14336, "block": 16,
         "out_dtype": "bf16"},
        # A decode step of 48 sequences through the up projection of a 70B model.
        {"name": "linear_batch", "kind": "linear", "rows": 48, "out": 28672, "in": 8192, "block": 16,
         "out_dtype": "bf16"},
        # A prompt of 4000 tokens through the gate projection, blocks of 32.
        {"name": "linear_prompt", "kind": "linear", "rows": 4000, "out": 14336, "in": 4096, "block": 32,
         "out_dtype": "bf16"},
        # The gradient that reaches the activation of the same projection when an adapter is trained.
        {"name": "linear_grad_step", "kind": "linear_grad", "rows": 4096, "out": 14336, "in": 4096,
         "format": "nvfp4", "block": 16, "out_dtype": "bf16"},
        # The gated block of an 8B model for four tokens: bound by its 235 MB of weights.
        {"name": "ffn_tokens", "kind": "ffn", "rows": 4, "out": 14336, "in": 4096, "save": False},
        # The same for a training step of 8192 tokens, keeping the pre-activations.
        {"name": "ffn_step", "kind": "ffn", "rows": 8192, "out": 14336, "in": 4096, "save": True},
        # Its backward pass for 4000 tokens.
        {"name": "ffn_grad_step", "kind": "ffn_grad", "rows": 4000, "out": 14336, "in": 4096},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, unit, lo, hi):
    """A width of a layer: a multiple of `unit`, spread over its logarithm."""
    return unit * _log_int(rng, max(1, lo // unit), hi // unit)


def draw(rng: random.Random):
    """One more case of the listed kinds, over the sizes, types and options they stand for."""
    kind = rng.choice(("mx_round_trip", "mx_linear", "mx_linear", "linear", "linear", "linear_grad",
                       "ffn", "ffn_grad"))
    odd = rng.random() < 0.3                           # widths that no tile or load divides
    if kind == "mx_round_trip":
        cols = _log_int(rng, 16, 14336) if odd else _width(rng, 32, 32, 14336)
        return {"kind": kind, "rows": _log_int(rng, 1, min(32768, MOST_ELEMENTS // cols)), "cols": cols,
                "dtype": rng.choice(("bf16", "f32"))}
    block = rng.choice((16, 16, 32, 64, 128)) if kind in ("linear", "linear_grad") else 8
    form = rng.choice(("nvfp4", "nvfp4", "mxfp4"))
    unit = 1 if odd and block == 8 else block
    k = _width(rng, unit, 128, 14336)
    n = _log_int(rng, 64, 28672) if odd else _width(rng, 16, 64, 28672)
    each = {"mx_linear": 2, "linear": 2, "linear_grad": 2, "ffn": 4, "ffn_grad": 8}[kind]
    most = max(1, min(8192, MOST_FLOPS // (each * n * k)))
    rows = _log_int(rng, min(64, most) if kind.endswith("grad") else 1, most)    # training has no single rows
    case = {"kind": kind, "rows": rows, "out": n, "in": k}
    if kind == "mx_linear":
        case.update(dtype=rng.choice(("bf16", "f32")), out_dtype=rng.choice(("bf16", "bf16", "f32")))
    elif kind == "linear":
        case.update(block=block, out_dtype=rng.choice(("bf16", "bf16", "f32")))
    elif kind == "linear_grad":
        case.update(format=form, block=32 if form == "mxfp4" else block,
                    out_dtype=rng.choice(("bf16", "bf16", "f32")))
        if form == "mxfp4":
            case["in"] = k if not odd else _log_int(rng, 128, k)
    elif kind == "ffn":
        case.update(save=rng.random() < 0.5)
    return case


# ---- inputs --------------------------------------------------------------------------------

def _weight(n, k, g):
    """[n, k] weight: 0.02 N(0, 1), every thousandth input column ten times as large."""
    w = torch.randn((n, k), generator=g, device=g.device).mul_(0.02)
    w[:, 7::1000] *= 10.0
    return w


def _activation(m, k, g):
    """[m, k] activation: N(0, 1), every 512th channel fifty times as large."""
    x = torch.randn((m, k), generator=g, device=g.device)
    x[:, 5::512] *= 50.0
    return x


def _codes(v):
    """E2M1 codes of v, to nearest, ties to the even code, saturating at 6."""
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for m, up in MIDPOINTS:
        code += (a >= m) if up else (a > m)
    return code + (torch.signbit(v).to(torch.uint8) << 3)


def _pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _nvfp4(w, block):
    """(nibbles, E4M3 codes, S) of w by the AbsMax rule."""
    n, k = w.shape
    S = (w.abs().max() / (448.0 * 6.0)).reshape(1)
    y = (w / S).view(n, k // block, block)
    s = (y.abs().amax(-1, keepdim=True) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    f = s.float()
    code = _codes(torch.where(f > 0, y / f.clamp(min=2.0 ** -9), torch.zeros_like(y)))
    return _pack(code.view(n, k)), s.view(torch.uint8).view(n, k // block), S


def _mxfp4(x):
    """(nibbles, E8M0 codes) of x: blocks of 32 along the rows, the last one filled up with zeros; the
    scale is 2^(floor(log2 max|x|) - 2), and the code 255 stands for a block with no finite maximum."""
    m, k = x.shape
    kb = (k + 31) // 32
    y = torch.nn.functional.pad(x.float(), (0, kb * 32 - k)).view(m, kb, 32)
    top = y.abs().amax(-1)
    ok = torch.isfinite(top)
    e = torch.where(ok & (top > 0), torch.frexp(top).exponent - 3, -127).clamp(-127, 127)
    code = _codes(torch.ldexp(y, -e.unsqueeze(-1)))
    return _pack(code.view(m, kb * 32)), torch.where(ok, e + 127, 255).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 17)
    kind = case["kind"]
    st = {"case": case}
    if kind == "mx_round_trip":
        st["x"] = _activation(case["rows"], case["cols"], g).to(DTYPES[case["dtype"]])
        return st
    m, n, k = case["rows"], case["out"], case["in"]
    if kind in ("ffn", "ffn_grad"):
        st["x"] = torch.randn((m, k), generator=g, device="cuda").to(torch.bfloat16)
        st["wg"] = _weight(n, k, g).to(torch.bfloat16)
        st["wu"] = _weight(n, k, g).to(torch.bfloat16)
        if kind == "ffn_grad":
            x = st["x"].float()
            st["g"] = (x @ st["wg"].float().t()).to(torch.bfloat16)
            st["u"] = (x @ st["wu"].float().t()).to(torch.bfloat16)
            st["dh"] = torch.randn((m, n), generator=g, device="cuda").to(torch.bfloat16)
        return st
    w = _weight(n, k, g)
    mx = kind == "mx_linear" or case.get("format") == "mxfp4"
    st["w"] = _mxfp4(w) if mx else _nvfp4(w, case["block"])
    if kind == "linear_grad":
        st["dy"] = torch.randn((m, n), generator=g, device="cuda").to(torch.bfloat16)
    else:
        st["x"] = _activation(m, k, g).to(DTYPES[case.get("dtype", "bf16")])
    return st


# ---- the operators in elementary operations --------------------------------------------------

def _unpack(q):
    """The E2M1 values of packed nibbles, low nibble first."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=q.device)
    both = torch.stack((q & 15, q >> 4), -1).view(q.shape[0], -1)
    return table[both.long()]


def _mx_values(q, scales):
    n = q.shape[0]
    s = torch.ldexp(torch.ones((), device=q.device), scales.int() - 127)
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return (_unpack(q).view(n, -1, 32) * s.unsqueeze(-1)).view(n, -1)


def _nvfp4_values(q, scales, S, block):
    n = q.shape[0]
    s = scales.view(torch.float8_e4m3fn).float()
    return (_unpack(q).view(n, -1, block) * s.unsqueeze(-1)).view(n, -1) * S


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "mx_round_trip":
        return _mx_values(*_mxfp4(st["x"]))[:, :case["cols"]].to(st["x"].dtype)
    if kind == "mx_linear":
        return (_mx_values(*_mxfp4(st["x"])) @ _mx_values(*st["w"]).t()).to(DTYPES[case["out_dtype"]])
    if kind == "linear":
        return (st["x"].float() @ _nvfp4_values(*st["w"], case["block"]).t()).to(DTYPES[case["out_dtype"]])
    if kind == "linear_grad":
        w = _mx_values(*st["w"])[:, :case["in"]] if case["format"] == "mxfp4" else \
            _nvfp4_values(*st["w"], case["block"])
        return (st["dy"].float() @ w).to(DTYPES[case["out_dtype"]])
    x, wg, wu = st["x"].float(), st["wg"].float(), st["wu"].float()
    if kind == "ffn":
        g, u = x @ wg.t(), x @ wu.t()
        h = (g / (1.0 + torch.exp(-g)) * u).to(torch.bfloat16)
        return (h, g.to(torch.bfloat16), u.to(torch.bfloat16)) if case["save"] else h
    g, u, dh = st["g"].float(), st["u"].float(), st["dh"].float()
    s = 1.0 / (1.0 + torch.exp(-g))
    dg = dh * u * s * (1.0 + g * (1.0 - s))
    du = dh * g * s
    return ((dg @ wg + du @ wu).to(torch.bfloat16), (dg.t() @ x).to(torch.bfloat16),
            (du.t() @ x).to(torch.bfloat16))


def run(state):
    if not own:
        return _plain(state)
    import paper_2606_07618_amd as nv

    case = state["case"]
    kind = case["kind"]
    if kind == "mx_round_trip":
        x = state["x"]
        q, scales = nv.mx_quantize(x)
        return nv.mx_dequant(q, scales, cols=case["cols"], out_dtype=x.dtype)
    if kind == "mx_linear":
        return nv.mx_matmul(nv.mx_quantize(state["x"]), state["w"], out_dtype=DTYPES[case["out_dtype"]])
    if kind == "linear":
        return nv.matmul(state["x"], *state["w"], block=case["block"], out_dtype=DTYPES[case["out_dtype"]])
    if kind == "linear_grad":
        if case["format"] == "mxfp4":
            return nv.mx_matmul_grad_input(state["dy"], *state["w"], cols=case["in"],
                                           out_dtype=DTYPES[case["out_dtype"]])
        return nv.matmul_grad_input(state["dy"], *state["w"], block=case["block"],
                                    out_dtype=DTYPES[case["out_dtype"]])
    if kind == "ffn":
        return nv.swiglu_ffn(state["x"], state["wg"], state["wu"], save=case["save"])
    return nv.swiglu_ffn_backward(state["dh"], state["x"], state["wg"], state["wu"], state["g"], state["u"])


def work(case):
    kind = case["kind"]
    if kind == "mx_round_trip":
        e = case["rows"] * case["cols"]
        return {"bytes": 2 * e * (2 if case["dtype"] == "bf16" else 4), "flops": 2 * e}
    m, n, k = case["rows"], case["out"], case["in"]
    if kind == "ffn":
        return {"bytes": 2 * (m * k + 2 * n * k + m * n * (3 if case["save"] else 1)), "flops": 4 * m * n * k}
    if kind == "ffn_grad":
        return {"bytes": 2 * (2 * m * k + 4 * n * k + 3 * m * n), "flops": 8 * m * n * k}
    size = {"bf16": 2, "f32": 4}
    block = 32 if kind == "mx_linear" else case["block"]
    w = n * (k // 2 + -(-k // block))
    if kind == "linear_grad":
        return {"bytes": 2 * m * n + w + m * k * size[case["out_dtype"]], "flops": 2 * m * n * k}
    return {"bytes": m * k * size[case.get("dtype", "bf16")] + w + m * n * size[case["out_dtype"]],
            "flops": 2 * m * n * k}


# ---- the operators from their definitions in 64 bits ------------------------------------------

def _grid64(q):
    """E2M1 values from the fields of each nibble: 0 and 0.5 below exponent 1, then (1 + m/2) 2^(e-1)."""
    nib = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.int32, device=q.device)
    nib[:, 0::2], nib[:, 1::2] = q.int() & 15, q.int() >> 4
    e, m = (nib >> 1) & 3, (nib & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2((e - 1).double()))
    return torch.where(nib >= 8, -v, v)


def _weights64(case, w):
    if case["kind"] == "mx_linear" or case.get("format") == "mxfp4":
        q, codes = w
        return _grid64(q) * torch.exp2(codes.double() - 127.0).repeat_interleave(32, 1)
    q, codes, S = w
    c = codes.int()
    e, m = (c >> 3) & 15, (c & 7).double()
    s = torch.where(e == 0, m * 2.0 ** -9, (8.0 + m) * torch.exp2((e - 10).double()))
    return _grid64(q) * s.repeat_interleave(case["block"], 1) * S.double()


def _microscaled64(x):
    """x rounded to microscaled FP4, in 64 bits: quanta of 2^(e-1) above the smallest binade, half to even."""
    m, k = x.shape
    kb = (k + 31) // 32
    y = torch.zeros((m, kb * 32), dtype=torch.float64, device=x.device)
    y[:, :k] = x.double()
    y = y.view(m, kb, 32)
    top = y.abs().amax(-1, keepdim=True)
    scale = torch.exp2((torch.frexp(top).exponent - 3).double().clamp(min=-127.0))
    v = y / scale
    quantum = torch.exp2((torch.frexp(v.abs()).exponent - 2).double().clamp(min=-1.0))
    v = (torch.round(v / quantum) * quantum).clamp(-6.0, 6.0)
    return (v * scale).view(m, kb * 32)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "mx_round_trip":
        return torch.cat([_microscaled64(part)[:, :case["cols"]] for part in st["x"].split(1024)])
    if kind == "mx_linear":
        return _microscaled64(st["x"]) @ _weights64(case, st["w"]).t()
    if kind == "linear":
        return st["x"].double() @ _weights64(case, st["w"]).t()
    if kind == "linear_grad":
        return (st["dy"].double() @ _weights64(case, st["w"]))[:, :case["in"]]
    x, wg, wu = st["x"].double(), st["wg"].double(), st["wu"].double()
    if kind == "ffn":
        g, u = x @ wg.t(), x @ wu.t()
        h = g * torch.sigmoid(g) * u
        return (h, g, u) if case["save"] else h
    g, u, dh = st["g"].double(), st["u"].double(), st["dh"].double()
    s = torch.sigmoid(g)
    dg = dh * u * (s + g * s * (1.0 - s))
    du = dh * (g * s)
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x
