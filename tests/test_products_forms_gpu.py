"""Every form of the products, output for output against sums in 64 bits, at the sizes of product_shapes.py."""
import importlib.util

import pytest
import torch

import plain64
import product_shapes

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


@pytest.fixture(scope="module")
def ref():
    """plain64 with its 64-bit sums on the device: these sizes are too large for the host."""
    spec = importlib.util.spec_from_file_location("device64", plain64.__file__)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    grid = mod.SIGNED.to(DEV)

    def nibbles(q):
        out = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.float64, device=DEV)
        out[:, 0::2], out[:, 1::2] = grid[(q & 15).long()], grid[(q >> 4).long()]
        return out

    def mx_values(q, scales):
        return nibbles(q) * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)

    mod.f64 = lambda t: t.detach().double()
    mod.nibbles, mod.mx_values = nibbles, mx_values
    mod.e4m3 = lambda codes: codes.view(torch.float8_e4m3fn).float().double()
    return mod


def gen(*key):
    g = torch.Generator(DEV)
    g.manual_seed(hash(key) % 2 ** 31)              # of whole numbers: the same in every run
    return g


def rand(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


def codes(shape, lo, hi, g):
    return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.uint8)


def nvfp4(n, k, block, g):
    return codes((n, k // 2), 0, 256, g), codes((n, k // block), 0, 127, g), torch.full((1,), 0.0371, device=DEV)


def mx(n, k, g):
    kb = -(-k // 32)
    q = codes((n, 16 * kb), 0, 256, g)
    if k % 32:
        tail = q.view(n, kb, 16)[:, -1]
        tail[:, -(-(k % 32) // 2):] = 0
        if k % 2:
            tail[:, k % 32 // 2] &= 15
    return q, codes((n, kb), 110, 140, g)


def scaled(want, bound, S):
    s = float(S.item())
    return want * s, bound * s + 2.0 ** -23 * want.abs() * s


def linear(nv, ref, m, n, k, block):
    g = gen(1, m, n, k, block)
    q, sc, S = nvfp4(n, k, block, g)
    x = rand((m, k), g)
    want = scaled(*ref.product(ref.f64(x), ref.nvfp4_values(q, sc, block)), S)
    for out in (BF16, F32):
        ref.check(nv.matmul(x, q, sc, S, block=block, out_dtype=out), *want, "y")


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["linear"])
def test_linear(nv, ref, m, n, k):
    linear(nv, ref, m, n, k, 16)


@pytest.mark.parametrize("m,n,k,block", product_shapes.LONG)
def test_linear_long(nv, ref, m, n, k, block):
    linear(nv, ref, m, n, k, block)


@pytest.mark.parametrize("m,n,k,block", product_shapes.FEW_LINEAR)
def test_linear_few(nv, ref, m, n, k, block):
    linear(nv, ref, m, n, k, block)


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["grad"])
def test_grad(nv, ref, m, n, k):
    g = gen(2, m, n, k)
    q, sc, S = nvfp4(n, k, 16, g)
    dy = rand((m, n), g)
    want = scaled(*ref.product(ref.f64(dy), ref.nvfp4_values(q, sc, 16).t()), S)
    for out in (BF16, F32):
        ref.check(nv.matmul_grad_input(dy, q, sc, S, out_dtype=out), *want, "dx")


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["mxgrad"])
def test_mx_grad(nv, ref, m, n, k):
    g = gen(3, m, n, k)
    b, dy = mx(n, k, g), rand((m, n), g)
    want = ref.product(ref.f64(dy), ref.mx_values(*b)[:, :k].t())
    for out in (BF16, F32):
        ref.check(nv.mx_matmul_grad_input(dy, *b, cols=k, out_dtype=out), *want, "dx")


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["mx"])
def test_mx(nv, ref, m, n, k):
    g = gen(4, m, n, k)
    a, b = mx(m, k, g), mx(n, k, g)
    want = ref.product(ref.mx_values(*a), ref.mx_values(*b))
    for out in (BF16, F32):
        ref.check(nv.mx_matmul(a, b, out_dtype=out), *want, "y")


def block_operands(m, n, k, *key):
    g = gen(5, m, n, k, *key)
    return rand((m, k), g), rand((n, k), g, k ** -0.5), rand((n, k), g, k ** -0.5), rand((m, n), g)


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["ffn"] + product_shapes.FEW_FFN)
def test_ffn(nv, ref, m, n, k):
    x, wg, wu, _ = block_operands(m, n, k)
    got = nv.swiglu_ffn(x, wg, wu, save=True)
    for a, want, bound, what in zip(got, *ref.ffn(x, wg, wu), ("h", "gate", "up")):
        ref.check(a, want, bound, what)
    assert torch.equal(nv.swiglu_ffn(x, wg, wu), got[0])


@pytest.mark.parametrize("m,n,k", product_shapes.SHAPES["dx"] + product_shapes.SHAPES["dw"])
def test_ffn_gradients(nv, ref, m, n, k):
    x, wg, wu, dh = block_operands(m, n, k, 1)
    gate, up = rand((m, n), gen(6, m, n, k), 2.0), rand((m, n), gen(7, m, n, k))
    got = nv.swiglu_ffn_backward(dh, x, wg, wu, gate, up)
    for a, want, bound, what in zip(got, *ref.ffn_grads(dh, x, wg, wu, gate, up), ("dx", "dw_gate", "dw_up")):
        ref.check(a, want, bound, what)
