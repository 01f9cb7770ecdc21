"""A quantized mixture-of-experts block as it is used: a projection in 8 bits, rows sorted by expert, the experts' gated
feed-forward layers in NVFP4 from one batched quantization each, and back to the tokens; forward and backward."""
import pytest
import torch

import plain64
import workloads

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
ROUND = 2.0 ** -8


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def rand(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def experts_of(nv, w):
    """(q, scales, S) of each of the matrices w, stacked."""
    return tuple(torch.cat([t if t.dim() == 1 else t.unsqueeze(0) for t in p])
                 for p in zip(*(nv.quantize(m, "scalesweep_mse", 16) for m in w)))


def values(w, e):
    return plain64.nvfp4_values(w[0][e], w[1][e], 16) * float(w[2][e])


def near(got, want, share):
    """Within `share` of the largest value of a row: roundings of the steps before, whose errors a product sums up."""
    off = (plain64.f64(got) - want).abs().amax(1)
    top = want.abs().amax(1)
    assert bool((off <= share * top + 1e-30).all()), float((off / top.clamp(min=1e-30)).max())


@pytest.mark.parametrize("tokens,experts,used", [(1, 4, 2), (24, 8, 2), (300, 4, 2)])
def test_block(nv, tokens, experts, used):
    g = workloads.generator(DEV, 801, tokens)
    d, f = 256, 384
    x = rand((tokens, d), g)
    proj = nv.int8_quantize(rand((d, d), g, d ** -0.5))
    gate, up = (experts_of(nv, [rand((f, d), g, d ** -0.5) for _ in range(experts)]) for _ in range(2))
    down = experts_of(nv, [rand((d, f), g, f ** -0.5) for _ in range(experts)])
    expert = torch.stack([torch.randperm(experts, generator=g, device=DEV)[:used] for _ in range(tokens)]).flatten()
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.bincount(expert, minlength=experts).cumsum(0)

    h = nv.int8_matmul(nv.int8_quantize(x), proj)
    rows = h[order // used].requires_grad_()
    a, b = nv.grouped_matmul(rows, offsets, *gate), nv.grouped_matmul(rows, offsets, *up)
    m = nv.swiglu(a.detach(), b.detach()).requires_grad_()
    y = nv.grouped_matmul(m, offsets, *down)
    out = torch.zeros((tokens, d), dtype=torch.float32, device=DEV).index_add_(0, order // used, y.detach().float())

    # each step against 64 bits from the step before as it was rounded
    pq, ps = (plain64.f64(t) for t in proj)
    xq, xs = (plain64.f64(t) for t in nv.int8_quantize(x))
    p64 = (xq @ pq.t()) * xs.unsqueeze(1) * ps            # the integers' sum first, which is exact
    want = p64
    plain64.check(h, want, 4 * 2.0 ** -24 * want.abs(), "h")
    who = expert[order].cpu()
    for got, w, src in ((a, gate, rows), (b, up, rows), (y, down, m)):
        for e in range(experts):
            mine = who == e
            if mine.any():
                want, bound = plain64.product(plain64.f64(src)[mine], values(w, e))
                plain64.check(got.detach().cpu()[mine], want, bound + 2.0 ** -22 * (plain64.f64(src)[mine].abs() @ values(w, e).abs().t()), "y")
    # the whole block: h, a, b, m and y are each rounded once, h's 8-bit operands are as they are
    whole = torch.zeros((tokens, d), dtype=torch.float64)
    for i in range(tokens * used):
        t, e = int(order[i]) // used, int(who[i])
        whole[t] += (plain64.silu(p64[t] @ values(gate, e).t()) * (p64[t] @ values(up, e).t())) @ values(down, e).t()
    near(out, whole, 16 * ROUND)

    # gradients: through the experts' products to the rows
    dy = rand(y.shape, g)
    y.backward(dy)
    for e in range(experts):
        mine = who == e
        if mine.any():
            want, bound = plain64.product(plain64.f64(dy)[mine], values(down, e).t())
            plain64.check(m.grad.cpu()[mine], want, bound + 2.0 ** -22 * (plain64.f64(dy)[mine].abs() @ values(down, e).abs()), "dm")
    da, db = rand(a.shape, g), rand(b.shape, g)
    torch.autograd.backward((a, b), (da, db))
    for e in range(experts):
        mine = who == e
        if mine.any():
            u, eu = plain64.product(plain64.f64(da)[mine], values(gate, e).t())
            v, ev = plain64.product(plain64.f64(db)[mine], values(up, e).t())
            # each gradient is rounded to bfloat16, then autograd adds them in bfloat16
            lim = eu + ev + (ROUND + 2.0 ** -20) * (u.abs() + v.abs() + eu + ev) * 1.01
            plain64.check(rows.grad.cpu()[mine], u + v, lim, "drows")
