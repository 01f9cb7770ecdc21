"""The layers of a quantized mixture-of-experts block beside the single NVFP4 products: dense layers in
8 bits and experts in NVFP4, as cases that can be timed and compared.

``run`` computes a case either in elementary torch operations in 32 bits (``own`` false) or through
the package's entry points (``own`` true).  The kinds:

  int8_linear    a linear layer in 8-bit integers: the activation is quantized with a scale for each
                 token, then multiplied with weights that have a scale for each output channel
  int8_grad      its gradient with respect to the activation
  experts        rows sorted by expert, each group times the NVFP4 weights of its own expert
  experts_grad   its gradient with respect to the rows
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
MOST_FLOPS = 1_900_000_000_000    # of a drawn case: the listed prompt through eight experts
MOST_WEIGHTS = 805_306_368        # of a drawn case's experts together: the listed 128 of [1536, 4096]


def listed():
    return [
        # One token through the gate projection of an 8B model in 8 bits: launches, then reading the weights.
        {"name": "int8_linear_token", "kind": "int8_linear", "rows": 1, "out": 14336, "in": 4096,
         "dtype": "bf16", "out_dtype": "bf16"},
        # A decode step of 48 sequences through the up projection of a 70B model.
        {"name": "int8_linear_batch", "kind": "int8_linear", "rows": 48, "out": 28672, "in": 8192,
         "dtype": "bf16", "out_dtype": "bf16"},
        # A prompt of 777 tokens through a down projection cut for a shard, rows of no whole 16 values,
        # sums kept in binary32 for a later reduction over shards: ragged in every direction.
        {"name": "int8_linear_ragged", "kind": "int8_linear", "rows": 777, "out": 1001, "in": 14330,
         "dtype": "f32", "out_dtype": "f32"},
        # A prompt of 8192 tokens through the gate projection of an 8B model.
        {"name": "int8_linear_prompt", "kind": "int8_linear", "rows": 8192, "out": 14336, "in": 4096,
         "dtype": "bf16", "out_dtype": "bf16"},
        # The gradient that reaches the activation of the same projection when an adapter is trained.
        {"name": "int8_grad_step", "kind": "int8_grad", "rows": 4096, "out": 14336, "in": 4096},
        # The same of a small layer with widths that no tile divides.
        {"name": "int8_grad_ragged", "kind": "int8_grad", "rows": 333, "out": 1001, "in": 1500},
        # One token through the gate projections of two of eight experts: two rows, and two experts' weights to read.
        {"name": "experts_token", "kind": "experts", "rows": 2, "spare": 0, "experts": 8, "out": 14336, "in": 4096,
         "block": 16, "skew": 0.0, "out_dtype": "bf16"},
        # A decode step of 64 sequences, eight of 128 small experts each: four rows an expert, and all the weights.
        {"name": "experts_batch", "kind": "experts", "rows": 512, "spare": 0, "experts": 128, "out": 1536, "in": 4096,
         "block": 16, "skew": 0.5, "out_dtype": "bf16"},
        # A short prompt in a batch filled up to 800 rows, routed very unevenly, blocks of 32, odd widths, in binary32.
        {"name": "experts_ragged", "kind": "experts", "rows": 777, "spare": 23, "experts": 16, "out": 1001, "in": 2080,
         "block": 32, "skew": 1.2, "out_dtype": "f32"},
        # A prompt of 8192 tokens, two of eight experts each, through the gate projections.
        {"name": "experts_prompt", "kind": "experts", "rows": 16384, "spare": 0, "experts": 8, "out": 14336, "in": 4096,
         "block": 16, "skew": 0.3, "out_dtype": "bf16"},
        # The gradient of the same for 4096 tokens, when what lies before the experts is trained.
        {"name": "experts_grad_step", "kind": "experts_grad", "rows": 8192, "spare": 0, "experts": 8, "out": 14336,
         "in": 4096, "block": 16, "skew": 0.3, "out_dtype": "bf16"},
        # A small step over 32 narrow experts, some of which get next to nothing, odd widths, in binary32.
        {"name": "experts_grad_ragged", "kind": "experts_grad", "rows": 1000, "spare": 24, "experts": 32, "out": 1001,
         "in": 1552, "block": 16, "skew": 1.0, "out_dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, unit, lo, hi):
    """A width of a layer: a multiple of `unit`, spread over its logarithm."""
    return unit * _log_int(rng, max(1, lo // unit), hi // unit)


def draw(rng: random.Random):
    """One more case of the listed kinds, over the sizes, types and options they stand for."""
    kind = rng.choice(("int8_linear", "int8_linear", "int8_grad", "experts", "experts", "experts", "experts_grad"))
    odd = rng.random() < 0.3                           # widths that no tile or load divides
    n = _log_int(rng, 64, 28672) if odd else _width(rng, 16, 64, 28672)
    if kind.startswith("int8"):
        k = _log_int(rng, 64, 14336) if odd else _width(rng, 16, 64, 14336)
        most = max(1, min(8192, MOST_FLOPS // (2 * n * k)))
        if kind == "int8_grad":
            return {"kind": kind, "rows": _log_int(rng, min(64, most), most), "out": n, "in": k}
        return {"kind": kind, "rows": _log_int(rng, 1, most), "out": n, "in": k, "dtype": rng.choice(("bf16", "f32")),
                "out_dtype": rng.choice(("bf16", "bf16", "f32"))}
    block = rng.choice((16, 16, 32, 64, 128))
    k = _width(rng, block, 128, 14336)
    experts = _log_int(rng, 2, max(2, min(128, MOST_WEIGHTS // (n * k))))
    case = {"kind": kind, "rows": 0, "spare": 0, "experts": experts, "out": n, "in": k, "block": block,
            "skew": rng.choice((0.0, 0.3, 0.6, 1.2)), "out_dtype": rng.choice(("bf16", "bf16", "f32"))}
    # every expert's rows as many as the fullest one's: what the plain form computes
    share = sum((e + 1) ** -case["skew"] for e in range(experts)) / experts
    most = max(1, min(16384, int(MOST_FLOPS * share / (2 * n * k))))
    case["rows"] = _log_int(rng, min(64, most) if kind == "experts_grad" else 1, most)
    if rng.random() < 0.3:
        case["spare"] = _log_int(rng, 1, 64)
    return case


def _sizes(case):
    """Rows of each expert, the fullest first: shares of 1 / (i + 1)^skew, whole rows by largest remainder."""
    share = [(e + 1) ** -case["skew"] for e in range(case["experts"])]
    exact_ = [case["rows"] * s / sum(share) for s in share]
    sizes = [int(v) for v in exact_]
    order = sorted(range(len(sizes)), key=lambda e: (sizes[e] - exact_[e], e))
    for e in order[:case["rows"] - sum(sizes)]:
        sizes[e] += 1
    return sizes


# ---- inputs --------------------------------------------------------------------------------

def _weight(shape, g):
    """[.., n, k] weights: 0.02 N(0, 1), every thousandth input column ten times as large."""
    w = torch.randn(shape, generator=g, device=g.device).mul_(0.02)
    w[..., 7::1000] *= 10.0
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


def _nvfp4(w, block):
    """(nibbles, E4M3 codes, S) of each of the matrices w by the AbsMax rule."""
    e, n, k = w.shape
    S = w.abs().amax((1, 2)) / (448.0 * 6.0)
    y = (w / S.view(e, 1, 1)).view(e, n, k // block, block)
    s = (y.abs().amax(-1, keepdim=True) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    f = s.float()
    code = _codes(torch.where(f > 0, y / f.clamp(min=2.0 ** -9), torch.zeros_like(y))).view(e, n, k)
    return code[..., 0::2] | (code[..., 1::2] << 4), s.view(torch.uint8).view(e, n, k // block), S


def _int8(x):
    """(q, scales) of the rows of x: scale = max|x| / 127 in binary32, q the nearest whole number to
    x / scale, ties to even (the quotient in 64 bits: next to a tie, 32 may land on it)."""
    x = x.float()
    s = x.abs().amax(-1) / 127.0
    y = x.double() / s.double().clamp(min=2.0 ** -149).unsqueeze(-1)
    return torch.round(y).clamp(-127.0, 127.0).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 29)
    kind, n, k = case["kind"], case["out"], case["in"]
    st = {"case": case}
    if kind.startswith("int8"):
        q, s = _int8(_weight((n, k), g))
        st["w"] = torch.nn.functional.pad(q, (0, -k % 16)), s        # rows of whole 16 values, as the package has them
        if kind == "int8_linear":
            st["x"] = _activation(case["rows"], k, g).to(DTYPES[case["dtype"]])
        else:
            st["dy"] = torch.randn((case["rows"], n), generator=g, device="cuda").to(torch.bfloat16)
        return st
    sizes = _sizes(case)
    random.Random(seed).shuffle(sizes)
    ends = [sum(sizes[:e]) for e in range(len(sizes) + 1)]
    st["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    st["fullest"] = max(sizes)
    parts = [_nvfp4(_weight((1, n, k), g), case["block"]) for _ in sizes]
    st["w"] = tuple(torch.cat(p) for p in zip(*parts))
    rows = case["rows"] + case["spare"]
    if kind == "experts":
        st["x"] = _activation(rows, k, g).to(torch.bfloat16)
    else:
        st["dy"] = torch.randn((rows, n), generator=g, device="cuda").to(torch.bfloat16)
    return st


# ---- the operators in elementary operations --------------------------------------------------

def _nvfp4_values(q, scales, S, block):
    """The values of packed nibbles, low nibble first, times their scales."""
    e, n = q.shape[:2]
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=q.device)
    v = table[torch.stack((q & 15, q >> 4), -1).view(e, n, -1).int()]
    s = scales.view(torch.float8_e4m3fn).float()
    return (v.view(e, n, -1, block) * s.unsqueeze(-1)).view(e, n, -1) * S.view(e, 1, 1)


def _by_expert(rows, offsets, fullest, w):
    """rows[i] @ w[expert of i]: each expert's rows filled up with zeros to as many as the fullest one's.
    Rows behind the last expert's give zeros."""
    experts = w.shape[0]
    at = torch.arange(rows.shape[0], dtype=torch.int32, device=rows.device)
    expert = torch.searchsorted(offsets[1:], at, right=True)
    inside = expert < experts
    expert = expert.clamp(max=experts - 1)
    place = torch.where(inside, at - offsets[expert], fullest)       # the others in a row of their own
    filled = rows.new_zeros((experts, fullest + 1, rows.shape[1]))
    filled[expert, place] = torch.where(inside.unsqueeze(1), rows, torch.zeros_like(rows))
    return torch.bmm(filled, w)[expert, place]


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "int8_linear":
        (a, sa), (b, sb) = _int8(st["x"]), st["w"]
        y = a.float() @ b[:, :case["in"]].float().t()
        return (y * sa.unsqueeze(1) * sb).to(DTYPES[case["out_dtype"]])
    if kind == "int8_grad":
        q, s = st["w"]
        return ((st["dy"].float() * s) @ q[:, :case["in"]].float()).to(torch.bfloat16)
    w = _nvfp4_values(*st["w"], case["block"])
    if kind == "experts":
        y = _by_expert(st["x"].float(), st["offsets"], st["fullest"], w.transpose(1, 2))
    else:
        y = _by_expert(st["dy"].float(), st["offsets"], st["fullest"], w)
    return y.to(DTYPES[case["out_dtype"]])


def run(state):
    if not own:
        return _plain(state)
    import paper_2606_07618_amd as nv

    case = state["case"]
    kind = case["kind"]
    if kind == "int8_linear":
        return nv.int8_matmul(nv.int8_quantize(state["x"]), state["w"], out_dtype=DTYPES[case["out_dtype"]])
    if kind == "int8_grad":
        return nv.int8_matmul_grad_input(state["dy"], *state["w"], cols=case["in"])
    product = nv.grouped_matmul if kind == "experts" else nv.grouped_matmul_grad_input
    return product(state["x" if kind == "experts" else "dy"], state["offsets"], *state["w"], block=case["block"],
                   out_dtype=DTYPES[case["out_dtype"]])


def work(case):
    kind, n, k = case["kind"], case["out"], case["in"]
    size = {"bf16": 2, "f32": 4}
    if kind == "int8_linear":
        m = case["rows"]
        return {"bytes": m * k * size[case["dtype"]] + n * k + 4 * n + m * n * size[case["out_dtype"]],
                "flops": 2 * m * n * k}
    if kind == "int8_grad":
        m = case["rows"]
        return {"bytes": 2 * m * n + n * k + 4 * n + 2 * m * k, "flops": 2 * m * n * k}
    m = case["rows"]
    active = sum(s > 0 for s in _sizes(case))
    inner, outer = (k, n) if kind == "experts" else (n, k)
    return {"bytes": 2 * m * inner + active * (n * k // 2 + n * k // case["block"] + 4)
            + (m + case["spare"]) * outer * size[case["out_dtype"]], "flops": 2 * m * n * k}


# ---- the operators from their definitions in 64 bits ------------------------------------------

def _grid64(q):
    """E2M1 values from the fields of each nibble: 0 and 0.5 below exponent 1, then (1 + m/2) 2^(e-1)."""
    nib = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.int32, device=q.device)
    nib[:, 0::2], nib[:, 1::2] = q.int() & 15, q.int() >> 4
    e, m = (nib >> 1) & 3, (nib & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2((e - 1).double()))
    return torch.where(nib >= 8, -v, v)


def _expert64(w, i, block):
    q, codes, S = w[0][i], w[1][i].int(), w[2][i]
    e, m = (codes >> 3) & 15, (codes & 7).double()
    s = torch.where(e == 0, m * 2.0 ** -9, (8.0 + m) * torch.exp2((e - 10).double()))
    return _grid64(q) * s.repeat_interleave(block, 1) * S.double()


def _int8_rows64(x):
    """The values of x as 8-bit integers times their row's scale: whole steps of the scale next to x, the
    even one where two are equally near."""
    x = x.double()
    s = (x.abs().amax(1, keepdim=True) / 127.0).float().double()     # the scale is held in binary32
    y = torch.where(s > 0, x / s, torch.zeros_like(x))
    low = torch.floor(y)
    up = (y - low > 0.5) | ((y - low == 0.5) & (low % 2 != 0))
    return (low + up) * s


def exact(case, seed):
    st = prepare(case, seed)
    kind, k = case["kind"], case["in"]
    if kind == "int8_linear":
        q, s = st["w"]
        w = q[:, :k].double() * s.double().unsqueeze(1)
        return torch.cat([_int8_rows64(part) @ w.t() for part in st["x"].split(2048)])
    if kind == "int8_grad":
        q, s = st["w"]
        return st["dy"].double() @ (q[:, :k].double() * s.double().unsqueeze(1))
    rows = st["x" if kind == "experts" else "dy"].double()
    y = torch.zeros((rows.shape[0], case["out"] if kind == "experts" else k), dtype=torch.float64, device=rows.device)
    ends = st["offsets"].tolist()
    for e in range(case["experts"]):
        if ends[e] < ends[e + 1]:
            w = _expert64(st["w"], e, case["block"])
            y[ends[e]:ends[e + 1]] = rows[ends[e]:ends[e + 1]] @ (w.t() if kind == "experts" else w)
    return y
