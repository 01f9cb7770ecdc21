"""Products of operands that require a gradient are recorded: their gradients are those of the gradient calls, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def rand(*shape, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).bfloat16()


def grads(outputs, inputs, d):
    return torch.autograd.grad(outputs, inputs, d, allow_unused=True)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k,block", [(1, 40, 64, 16), (40, 96, 512, 32), (600, 77, 208, 16)])
def test_matmul(nv, m, n, k, block, out):
    w = nv.quantize(rand(n, k, seed=1), "scalesweep_mse", block)
    x, dy = rand(m, k).requires_grad_(), rand(m, n, seed=2)
    y = nv.matmul(x, *w, block=block, out_dtype=out)
    assert y.requires_grad and torch.equal(y.detach(), nv.matmul(x.detach(), *w, block=block, out_dtype=out))
    dx, = grads(y, x, dy.to(out))
    assert torch.equal(dx, nv.matmul_grad_input(dy, *w, block=block))


def test_gradients_in_any_layout(nv):
    """One value for all of dy, a dy whose rows start anywhere, one whose columns are rows."""
    m, n, k = 12, 39, 64
    w = nv.quantize(rand(n, k, seed=1), "absmax")
    x = rand(m, k).requires_grad_()
    whole = rand(m + 1, n, seed=3)
    for dy in (whole[:1, :1].expand(m, n), whole[1:], rand(n, m, seed=4).t()):
        dx, = grads(nv.matmul(x, *w), x, dy)
        assert torch.equal(dx, nv.matmul_grad_input(dy.clone(memory_format=torch.contiguous_format), *w))


@pytest.mark.parametrize("m,n,k", [(1, 40, 64), (70, 96, 71), (300, 77, 208)])
def test_swiglu_ffn(nv, m, n, k):
    x, wg, wu, dh = rand(m, k), rand(n, k, seed=1), rand(n, k, seed=2), rand(m, n, seed=3)
    h, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
    want = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up)
    for needs in ((1, 1, 1), (1, 0, 0), (0, 1, 1), (0, 0, 1)):
        args = [t.clone().requires_grad_(bool(need)) for t, need in zip((x, wg, wu), needs)]
        got = nv.swiglu_ffn(*args)
        assert torch.equal(got.detach(), h)
        got.backward(dh)
        for a, b, need in zip(args, want, needs):
            assert torch.equal(a.grad, b) if need else a.grad is None


def test_through_both(nv):
    """A gated block and a quantized projection behind a residual: every operand gets its gradient."""
    m, n, k = 33, 128, 64
    x, wg, wu = (rand(*s, seed=i).requires_grad_() for i, s in enumerate(((m, k), (n, k), (n, k))))
    down = nv.quantize(rand(k, n, seed=5), "scalesweep_mse")
    y = x + nv.matmul(nv.swiglu_ffn(x, wg, wu), *down)
    dy = rand(m, k, seed=6)
    y.backward(dy)
    with torch.no_grad():
        h, gate, up = nv.swiglu_ffn(x, wg, wu, save=True)
        dx, dwg, dwu = nv.swiglu_ffn_backward(nv.matmul_grad_input(dy, *down), x, wg, wu, gate, up)
        assert torch.equal(x.grad, dy + dx) and torch.equal(wg.grad, dwg) and torch.equal(wu.grad, dwu)


def test_what_is_not_recorded(nv):
    """No gradient wanted, the caller's own buffers, the caller's own backward."""
    m, n, k = 8, 32, 64
    w = nv.quantize(rand(n, k, seed=1), "absmax")
    x, wg = rand(m, k).requires_grad_(), rand(n, k, seed=2)
    buf = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    with torch.no_grad():
        assert not nv.matmul(x, *w).requires_grad and not nv.swiglu_ffn(x, wg, wg).requires_grad
    assert not nv.matmul(x.detach(), *w).requires_grad and not nv.swiglu_ffn(x.detach(), wg, wg).requires_grad
    assert not nv.matmul(x, *w, out=buf).requires_grad and not nv.swiglu_ffn(x, wg, wg, out=buf).requires_grad
    assert not any(t.requires_grad for t in nv.swiglu_ffn(x, wg, wg, save=True))


def test_second_derivatives_are_refused(nv):
    x, w = rand(8, 64).requires_grad_(), nv.quantize(rand(32, 64, seed=1), "absmax")
    dy = rand(8, 32, seed=2).requires_grad_()
    dx, = torch.autograd.grad(nv.matmul(x, *w), x, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()
