"""A binary32 gradient of an 8-bit product takes the weights s q whole: with bfloat16 operands in their place it was off by
up to 2^-9 of each term."""
import pytest
import torch

import plain64
import product_shapes
import workloads

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
U = 2.0 ** -24


@pytest.fixture(scope="module")
def nv():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2606_07618_amd as nv
    return nv


def gen(*key):
    return workloads.generator(DEV, 703, *key)


def weights(n, k, g):
    q = torch.randint(-128, 128, (n, -(-k // 16) * 16), generator=g, device=DEV, dtype=torch.int8)
    q[:, k:] = 0
    return q, torch.rand((n,), generator=g, device=DEV) * 0.1 + 1e-3


# every tile, whole and split, rows of whole chunks and not
SHAPES = [(1, 1, 16), (3, 7, 33), (64, 256, 512), (65, 130, 272), (200, 1001, 47)] + product_shapes.SHAPES["grad"]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_single_weights_come_back_whole(nv, m, n, k):
    """Rows of dy with a single one: each output is one weight, rounded where s q becomes a binary32 number and nowhere else."""
    g = gen(1, m, n, k)
    q, s = weights(n, k, g)
    at = torch.randint(0, n, (m,), generator=g, device=DEV)
    dy = torch.zeros((m, n), dtype=torch.bfloat16, device=DEV)
    dy[torch.arange(m, device=DEV), at] = 1.0
    got = nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32)
    assert torch.equal(got, (q[:, :k].float() * s.unsqueeze(1))[at])


@pytest.mark.parametrize("m,n,k", [s for s in SHAPES if s[0] * s[1] * s[2] < 2e9])
def test_sums(nv, m, n, k):
    g = gen(2, m, n, k)
    q, s = weights(n, k, g)
    dy = torch.randn((m, n), generator=g, device=DEV).to(torch.bfloat16)
    want, bound = plain64.product(plain64.f64(dy), (plain64.f64(q) * plain64.f64(s).unsqueeze(1))[:, :k].t())
    size = plain64.f64(dy).abs() @ (plain64.f64(q).abs() * plain64.f64(s).unsqueeze(1))[:, :k]
    # a sum for each of a weight's three numbers, the later ones of at most 2^-7 and 2^-14 of it; s q as a binary32 number; the
    # sums' two additions, the last of which check() counts
    got = nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32)
    plain64.check(got, want, 1.01 * bound + U * size + U * (want.abs() + bound), "dx")


def test_scales_of_every_size(nv):
    """From 2^-100, whose weights' last bits are still bfloat16 numbers, to binary32's largest weight."""
    g = gen(3)
    q, _ = weights(64, 96, g)
    s = torch.exp2(torch.linspace(-100, 120.9, 64, device=DEV)).float()
    q[:, 0] = 127
    dy = torch.eye(64, dtype=torch.bfloat16, device=DEV)
    want = q.float() * s.unsqueeze(1)
    assert bool(want.isfinite().all())
    assert torch.equal(nv.int8_matmul_grad_input(dy, q, s, out_dtype=torch.float32), want)


def test_infinite_weights_stay_infinite(nv):
    g = gen(4)
    q, s = weights(32, 48, g)
    q[5], s[5] = 127, 3e38
    dy = torch.zeros((40, 32), dtype=torch.bfloat16, device=DEV)
    dy[3, 5], dy[4, 5] = 1.0, -2.0
    got = nv.int8_matmul_grad_input(dy[3:5].contiguous(), q, s, out_dtype=torch.float32)
    assert bool((got[0] == float("inf")).all()) and bool((got[1] == -float("inf")).all())


@pytest.mark.parametrize("m,n,k", [(70, 200, 320), (137, 619, 11216)])
def test_own_buffers_captured_and_replayed(nv, m, n, k):
    """The output and the weights' buffer are written three times: a workspace of bytes that are no numbers, and replays."""
    g = gen(5, m)
    q, s = weights(n, k, g)
    dy = torch.randn((m, n), generator=g, device=DEV).to(torch.bfloat16)
    out = torch.full((m, k), float("nan"), device=DEV)
    need = nv.int8_product_grad_input_workspace_bytes(m, n, k, n)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    want = nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32)
    assert nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32, out=out, ws=ws) is out
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32, out=out, ws=ws)
    for _ in range(3):
        dy.copy_(torch.randn((m, n), generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32))


@pytest.mark.parametrize("m,k", [(3, 48), (70, 100)])
def test_no_outputs_of_the_layer(nv, m, k):
    """Nothing to sum: zeros, also on top of what the output held."""
    q, s = weights(0, k, gen(6))
    out = torch.full((m, k), float("nan"), device=DEV)
    dy = torch.empty((m, 0), dtype=torch.bfloat16, device=DEV)
    assert not nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32, out=out).any()


@pytest.mark.parametrize("m,n,k", [(3, 7, 33), (64, 256, 512), (137, 619, 11216)])
def test_infinite_and_no_numbers_of_dy(nv, m, n, k):
    """As with the weights themselves: a weight that is one bfloat16 number has no part that is zero, whose product would be none."""
    g = gen(7, m, n, k)
    q, s = weights(n, k, g)
    s[0] = 0.25                                           # powers of two among its weights
    q[0, :8] = torch.tensor([1, 2, 64, -128, 3, -1, 0, 127], dtype=torch.int8, device=DEV)
    dy = torch.randn((m, n), generator=g, device=DEV).to(torch.bfloat16)
    dy[0, 0], dy[1, 0], dy[m - 1, n - 1] = float("inf"), -float("inf"), float("nan")
    got = nv.int8_matmul_grad_input(dy, q, s, cols=k, out_dtype=torch.float32)
    sign = q[0, :k].float().sign()
    want = torch.where(sign == 0, torch.full_like(sign, float("nan")), sign * float("inf"))
    for row, w in ((0, want), (1, -want)):
        assert bool((got[row].isnan() == w.isnan()).all()) and torch.equal(got[row][sign != 0], w[sign != 0])
    assert bool(got[m - 1].isnan().all()) and bool(got[2:m - 1].isfinite().all())
