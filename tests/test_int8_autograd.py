"""8-bit integers and autograd: an activation that requires a gradient is not dropped from the graph without a word, and the
product's gradient reaches it straight through the quantization."""
import pytest
import torch

import plain64
import workloads

DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


def refused(nv, x):
    with pytest.raises(ValueError, match="requires a gradient"):
        nv.int8_quantize(x)


def test_an_input_that_requires_a_gradient_is_refused(nv):
    x = torch.ones((4, 32), requires_grad=True)
    refused(nv, x)
    refused(nv, x * 2)
    refused(nv, x.to(torch.bfloat16))
    for y in (x.detach(), torch.ones(4, 32)):            # what is refused next is the host's memory
        with pytest.raises(ValueError, match="device tensor"):
            nv.int8_quantize(y)
    with torch.no_grad(), pytest.raises(ValueError, match="device tensor"):
        nv.int8_quantize(x)


class Projection(torch.autograd.Function):
    """A layer of weights in 8-bit integers, as a program builds one."""
    @staticmethod
    def forward(ctx, nv, x, q, scales, cols):
        ctx.save_for_backward(q, scales)
        ctx.nv, ctx.cols = nv, cols
        return nv.int8_matmul(nv.int8_quantize(x), (q, scales))

    @staticmethod
    def backward(ctx, dy):
        return (None, ctx.nv.int8_matmul_grad_input(dy.contiguous(), *ctx.saved_tensors, cols=ctx.cols)) + (None,) * 3


@pytest.mark.gpu
def test_device_inputs(nv):
    x = torch.ones((4, 32), device=DEV, requires_grad=True)
    refused(nv, x)
    refused(nv, x + 1)
    q, s = nv.int8_quantize(x.detach())
    with torch.no_grad():
        r, t = nv.int8_quantize(x)
    assert torch.equal(q, r) and torch.equal(s, t) and not s.requires_grad


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,d,f,experts", [(1, 64, 48, 2), (40, 250, 96, 4), (300, 256, 384, 3)])
def test_gradient_through_experts_and_projection(nv, tokens, d, f, experts):
    """x -> a projection in 8 bits -> each token's expert, and x a second time beside them: both of its terms arrive."""
    g = workloads.generator(DEV, 707, tokens)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)

    wide = -(-d // 16) * 16                              # the experts' inputs are whole blocks
    x = rand(tokens, d).requires_grad_()
    proj = nv.int8_quantize(rand(wide, d) * d ** -0.5)
    parts = [nv.quantize(rand(f, wide) * wide ** -0.5, "scalesweep_mse", 16) for _ in range(experts)]
    w = tuple(torch.cat([t if t.dim() == 1 else t.unsqueeze(0) for t in p]) for p in zip(*parts))
    expert = torch.randint(0, experts, (tokens,), generator=g, device=DEV)
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = torch.bincount(expert, minlength=experts).cumsum(0)

    h = Projection.apply(nv, x, *proj, d)
    h.retain_grad()
    y = nv.grouped_matmul(h[order], offsets, *w)
    dy = rand(tokens, f)
    direct = rand(tokens, d)
    torch.autograd.backward((y, x), (dy, direct))

    # dy's rows -> the gradient of h, rounded once
    dh = torch.zeros((tokens, wide), dtype=torch.float64)
    lim = torch.zeros_like(dh)
    who, back = expert[order].cpu(), order.cpu()
    for e in range(experts):
        mine = who == e
        if mine.any():
            v = plain64.nvfp4_values(w[0][e], w[1][e], 16) * float(w[2][e])
            want, bound = plain64.product(plain64.f64(dy)[mine], v.t())
            dh[back[mine]] = want
            lim[back[mine]] = bound + 2.0 ** -22 * (plain64.f64(dy)[mine].abs() @ v.abs())
    plain64.check(h.grad, dh, lim, "dh")
    # the gradient of h as it was rounded -> x: weights rounded as operands, the product rounded, the two terms' sum rounded
    v = (plain64.f64(proj[0]) * plain64.f64(proj[1]).unsqueeze(1))[:, :d]
    want, bound = plain64.product(plain64.f64(h.grad), v.t())
    bound = 1.01 * bound + (2.0 ** -8 + 2.0 ** -23) * (plain64.f64(h.grad).abs() @ v.abs())
    first = bound + 2.0 ** -8 * (want.abs() + bound)
    plain64.check(x.grad, want + plain64.f64(direct), first, "dx")
