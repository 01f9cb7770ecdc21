"""The gated feed-forward block and its gradients against their formulas in 64 bits."""
import pytest
import torch

import plain64
import workloads

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def operands(m, n, k, *key, spread=1.0):
    g = workloads.generator(DEV, 521, m, n, k, *key)
    x = torch.randn((m, k), generator=g, device=DEV).to(torch.bfloat16)
    wg = (torch.randn((n, k), generator=g, device=DEV) * spread / max(k, 1) ** 0.5).to(torch.bfloat16)
    wu = (torch.randn((n, k), generator=g, device=DEV) / max(k, 1) ** 0.5).to(torch.bfloat16)
    dh = torch.randn((m, n), generator=g, device=DEV).to(torch.bfloat16)
    return x, wg, wu, dh


SHAPES = [(m, n, k) for m in (1, 2, 4, 8, 15, 16, 17, 33, 64, 65, 128, 130, 257) for n, k in ((77, 200), (256, 512))] + \
    [(1, 1, 1), (3, 130, 7), (40, 33, 129), (300, 520, 65), (1, 64, 4096), (16, 300, 2048), (513, 100, 64), (7, 1000, 1031)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(nv, m, n, k):
    x, wg, wu, _ = operands(m, n, k)
    want, bound = plain64.ffn(x, wg, wu)
    got = nv.swiglu_ffn(x, wg, wu, save=True)
    for a, b, c, what in zip(got, want, bound, ("h", "gate", "up")):
        plain64.check(a, b, c, what)
    assert torch.equal(nv.swiglu_ffn(x, wg, wu), got[0])


def test_wide_gates(nv):
    """Gates from far below where e^-g overflows to far above where it vanishes."""
    x, wg, wu, dh = operands(70, 96, 64, 1, spread=60.0)
    want, bound = plain64.ffn(x, wg, wu)
    assert float(want[1].max()) > 120 and float(want[1].min()) < -120
    h, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    plain64.check(h, want[0], bound[0] + 1e-35, "h")
    want, bound = plain64.ffn_grads(dh, x, wg, wu, g, u)
    for a, b, c in zip(nv.swiglu_ffn_backward(dh, x, wg, wu, g, u), want, bound):
        plain64.check(a, b, c + 1e-35, "gradient")


GRADS = [(1, 1, 1), (1, 64, 128), (7, 77, 200), (64, 256, 512), (65, 130, 129), (130, 33, 264), (300, 520, 64),
         (257, 200, 31), (513, 64, 96), (40, 1000, 48)]


@pytest.mark.parametrize("m,n,k", GRADS)
def test_gradients(nv, m, n, k):
    x, wg, wu, dh = operands(m, n, k, 2)
    _, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    want, bound = plain64.ffn_grads(dh, x, wg, wu, g, u)
    got = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u)
    for a, b, c, what in zip(got, want, bound, ("dx", "dw_gate", "dw_up")):
        plain64.check(a, b, c, what)
    dx, none, none2 = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u, need_w=False)
    assert none is None and none2 is None and torch.equal(dx, got[0])
    none, dwg, dwu = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u, need_x=False)
    assert none is None and torch.equal(dwg, got[1]) and torch.equal(dwu, got[2])


def test_gradients_by_differences(nv):
    """Central differences of <r, h> in 64 bits against the kernels' gradients.  The formulas are smooth on a
    scale of 1, so a step of 1e-4 leaves an error of 1e-8 of the third derivative, far below the bounds."""
    m, n, k = 12, 40, 24
    x, wg, wu, r = operands(m, n, k, 3)
    X, G, U, R = map(plain64.f64, (x, wg, wu, r))
    # pre-activations rounded as the forward stores them: a term of the bound, |d gradient / d g| < 1 each
    _, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    got = nv.swiglu_ffn_backward(r, x, wg, wu, g, u)
    exact, _ = plain64.ffn_grads(r, x, wg, wu, X @ G.t(), X @ U.t())
    _, bound = plain64.ffn_grads(r, x, wg, wu, g, u)

    def loss(x, g, u):
        return float((plain64.silu(x @ g.t()) * (x @ u.t()) * R).sum())

    eps = 1e-4
    args = [X, G, U]
    for which, grad in enumerate(exact):
        for at in ((0, 0), (5, 7), (grad.shape[0] - 1, k - 1)):
            lo, hi = [t.clone() for t in args], [t.clone() for t in args]
            lo[which][at] -= eps
            hi[which][at] += eps
            diff = (loss(*hi) - loss(*lo)) / (2 * eps)
            assert abs(diff - float(grad[at])) <= 1e-6 * max(1.0, abs(diff))
    # the kernels' gradients: the formula's at the stored pre-activations, which are 2^-8 of |g| and |u| away
    dg_g = (R.abs() * (X @ U.t()).abs() * (X @ G.t()).abs() + R.abs() * (X @ U.t()).abs()) * 2.0 ** -8
    du_g = (R.abs() * (X @ G.t()).abs()) * 1.1 * 2.0 ** -8
    extra = (dg_g @ G.abs() + du_g @ U.abs(), dg_g.t() @ X.abs(), du_g.t() @ X.abs())
    for a, b, c, e, what in zip(got, exact, bound, extra, ("dx", "dw_gate", "dw_up")):
        plain64.check(a, b, c + e, what)


@pytest.mark.parametrize("m", [1, 16, 40, 200])
@pytest.mark.parametrize("k", [136, 71])
def test_rows_between_nans(nv, m, k):
    """Strided rows in a storage of NaN: nothing outside the operands enters."""
    n = 90
    x, wg, wu, dh = operands(m, n, k, 4)
    views = [plain64.between_nans(t) for t in (x, wg, wu)]
    h, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    for a, b in zip((h, g, u), nv.swiglu_ffn(*views, save=True)):
        assert torch.equal(a, b)
    for a, b in zip(nv.swiglu_ffn_backward(dh, x, wg, wu, g, u), nv.swiglu_ffn_backward(dh, *views, g, u)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("m", [3, 40, 150])
def test_nan_and_infinity_stay_in_their_row(nv, m):
    x, wg, wu, dh = operands(m, 60, 72, 5)
    clean, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    dx = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u, need_w=False)[0]
    x[m - 1, 3] = float("nan")
    x[0, 7] = float("inf")
    got = nv.swiglu_ffn(x, wg, wu)
    assert bool(got[m - 1].isnan().all())
    assert torch.equal(got[1:m - 1], clean[1:m - 1])
    dh[0, 5] = float("nan")
    got = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u, need_w=False)[0]
    assert bool(got[0].isnan().all()) and torch.equal(got[1:], dx[1:])


@pytest.mark.parametrize("m,n,k", [(0, 32, 64), (8, 0, 64), (8, 32, 0)])
def test_empty(nv, m, n, k):
    x, wg, wu, dh = operands(m, n, k)
    h, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    assert h.shape == g.shape == u.shape == (m, n) and not h.any() and not g.any() and not u.any()
    dx, dwg, dwu = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u)
    assert dx.shape == (m, k) and dwg.shape == dwu.shape == (n, k)
    assert not dx.any() and not dwg.any() and not dwu.any()


@pytest.mark.parametrize("m", [1, 40, 200])
def test_other_stream_and_own_buffers(nv, m):
    x, wg, wu, dh = operands(m, 200, 520, 6)
    want = nv.swiglu_ffn(x, wg, wu, save=True)
    grads = nv.swiglu_ffn_backward(dh, x, wg, wu, want[1], want[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = tuple(torch.full_like(t, float("nan")) for t in want)
    gout = tuple(torch.full_like(t, float("nan")) for t in grads)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = x * 1
        for _ in range(20):
            late = late * 1
        nv.swiglu_ffn(late, wg, wu, save=True, out=out)
        nv.swiglu_ffn_backward(dh, late, wg, wu, out[1], out[2], out=gout)
    side.synchronize()
    for a, b in zip(want + grads, out + gout):
        assert torch.equal(a, b)


def test_long_offsets(nv):
    """Rows whose bytes pass 2^32 in x, h and dx."""
    k, m = 8192, 2 ** 18 + 300
    x0, wg, wu, dh0 = operands(300, 40, k, 7)
    x = torch.zeros((m, k), dtype=torch.bfloat16, device=DEV)
    x[-300:] = x0
    h, g, u = nv.swiglu_ffn(x, wg, wu, save=True)
    want, bound = plain64.ffn(x0, wg, wu)
    plain64.check(h[-300:], want[0], bound[0], "h")
    assert not bool(h[:-300].any())
    dh = torch.zeros((m, 40), dtype=torch.bfloat16, device=DEV)
    dh[-300:] = dh0
    dx = nv.swiglu_ffn_backward(dh, x, wg, wu, g, u, need_w=False)[0]
    want, bound = plain64.ffn_grads(dh0, x0, wg, wu, g[-300:], u[-300:])
    plain64.check(dx[-300:], want[0], bound[0], "dx")
    assert not bool(dx[:-300].any())
