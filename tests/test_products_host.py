"""Refusals of the products' C entry points and of their Python wrappers, on the host: validation returns
before any launch.  Made-up device addresses only where no GPU is visible, as a call that wrongly passed
would launch on them."""
import ctypes
import re
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parents[1]
P = ctypes.c_void_p
A = P(0x100000)                       # never dereferenced
OFF8, OFF2 = P(0x100008), P(0x100002)
BIG = 1 << 62

fake_pointers = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                   reason="made-up device addresses only where no GPU is visible")


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


def test_every_declared_symbol_is_exported_and_bound(nv):
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "nvfp4ss.h").read_text(), flags=re.S)
    names = set(re.findall(r"\b(mxfp4_\w+|nvfp4_\w*matmul\w*|nvfp4_swiglu_ffn\w*)\s*\(", text))
    assert len(names) == 14
    for n in names:
        assert hasattr(nv.lib, n) and getattr(nv, n).argtypes is not None, n


@fake_pointers
def test_mx_quant(nv):
    def call(x=A, dtype=1, rows=4, cols=70, q=A, sc=A):
        return nv.mxfp4_quant(x, dtype, rows, cols, q, sc, None)

    assert call(x=None) == call(q=None) == call(sc=None) == -1
    assert call(rows=-1) == call(cols=-1) == call(rows=BIG) == call(cols=(1 << 63) - 1) == -2
    assert call(dtype=2) == -4
    assert call(x=OFF8) == call(q=OFF8) == -7
    assert call(rows=0, x=None) == call(cols=0, q=None) == 0

    def back(q=A, sc=A, rows=4, cols=70, dtype=0, out=A):
        return nv.mxfp4_dequant(q, sc, rows, cols, dtype, out, None)

    assert back(q=None) == back(sc=None) == back(out=None) == -1
    assert back(rows=-1) == back(cols=-1) == back(rows=BIG) == -2
    assert back(dtype=7) == -4
    assert back(q=OFF8) == back(out=OFF8) == -7
    assert back(rows=0, out=None) == 0


@fake_pointers
def test_matmul(nv):
    def call(x=A, ldx=64, q=A, sc=A, block=16, S=A, m=4, n=8, k=64, dtype=1, out=A, ws=A, wsb=1 << 40):
        return nv.nvfp4_matmul(x, ldx, q, sc, block, S, m, n, k, dtype, out, ws, wsb, None)

    assert call(x=None) == call(q=None) == call(sc=None) == call(S=None) == call(out=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-64) == call(k=72) == call(ldx=56) == call(ldx=1 << 22) == -2
    assert call(n=(1 << 20) + 1) == call(k=1 << 21, ldx=1 << 21) == call(m=BIG) == -2
    assert call(block=24) == call(block=0) == -3
    assert call(dtype=2) == -4
    assert call(x=OFF8) == call(q=OFF8) == call(out=OFF8) == call(S=OFF2) == call(ldx=68) == -7
    need = nv.nvfp4_matmul_workspace_bytes(2000, 512, 512)
    assert need > 0
    big = dict(m=2000, n=512, k=512, ldx=512)
    assert call(ws=None, **big) == call(wsb=need - 1, **big) == -6
    assert call(ws=P(0x100010), **big) == -7
    assert call(m=0, x=None) == call(n=0, out=None) == 0
    assert nv.nvfp4_matmul_workspace_bytes(-1, 8, 64) == -2


@fake_pointers
@pytest.mark.parametrize("mx", [False, True])
def test_grad_input(nv, mx):
    def call(dy=A, ld=40, q=A, sc=A, block=16, S=A, m=4, n=40, k=64, dtype=1, out=A, ws=A, wsb=1 << 40):
        if mx:
            return nv.mxfp4_matmul_grad_input(dy, ld, q, sc, m, n, k, dtype, out, ws, wsb, None)
        return nv.nvfp4_matmul_grad_input(dy, ld, q, sc, block, S, m, n, k, dtype, out, ws, wsb, None)

    size = nv.mxfp4_matmul_grad_input_workspace_bytes if mx else nv.nvfp4_matmul_grad_input_workspace_bytes
    assert call(dy=None) == call(q=None) == call(sc=None) == call(out=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-64) == call(ld=39) == call(ld=1 << 22) == -2
    assert call(dtype=2) == -4
    assert call(dy=OFF8) == call(q=OFF8) == call(out=OFF8) == -7
    if not mx:
        assert call(block=20) == -3 and call(k=72) == -2 and call(S=None) == -1
    need = size(200, 510, 512, 510)
    assert need >= 200 * 512 * 2                       # rows of 510 values are copied to rows of 512
    big = dict(m=200, n=510, k=512, ld=510)
    assert call(ws=None, **big) == call(wsb=need - 1, **big) == -6
    assert call(ws=P(0x100010), **big) == -7
    assert call(m=0, dy=None) == call(k=0, out=None) == 0
    assert size(8, -1, 64, 64) == -2


@fake_pointers
def test_mx_matmul(nv):
    def call(aq=A, asc=A, bq=A, bsc=A, m=4, n=8, k=60, dtype=1, out=A, ws=A, wsb=1 << 40):
        return nv.mxfp4_matmul(aq, asc, bq, bsc, m, n, k, dtype, out, ws, wsb, None)

    assert call(aq=None) == call(asc=None) == call(bq=None) == call(bsc=None) == call(out=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-1) == call(n=1 << 21) == -2
    assert call(dtype=-1) == -4
    assert call(aq=OFF8) == call(bq=OFF8) == call(out=OFF8) == call(asc=OFF2) == call(bsc=OFF2) == -7
    need = nv.mxfp4_matmul_workspace_bytes(200, 80, 96)
    assert need > 0
    assert call(m=200, n=80, k=96, wsb=need - 1) == -6
    assert call(m=0, aq=None) == call(n=0, out=None) == 0


@fake_pointers
def test_swiglu_ffn(nv):
    def call(x=A, ldx=64, wg=A, wu=A, ldw=64, m=4, n=8, k=64, h=A, g=None, u=None, ws=None, wsb=0):
        return nv.nvfp4_swiglu_ffn(x, ldx, wg, wu, ldw, m, n, k, h, g, u, ws, wsb, None)

    assert call(x=None) == call(wg=None) == call(wu=None) == call(h=None) == call(g=A) == call(u=A) == -1
    assert call(m=-1) == call(n=-1) == call(k=-1) == call(ldx=63) == call(ldw=63) == call(ldw=1 << 22) == -2
    assert call(x=OFF8) == call(wg=OFF8) == call(wu=OFF8) == call(h=OFF8) == call(g=OFF8, u=A) == -7
    need = nv.nvfp4_swiglu_ffn_workspace_bytes(4, 8, 63, 63, 63)
    assert need > 0
    odd = dict(k=63, ldx=63, ldw=63)
    assert call(**odd) == call(ws=A, wsb=need - 1, **odd) == -6
    assert call(ws=P(0x100010), wsb=need, **odd) == -7
    assert call(m=0, x=None) == call(n=0, h=None) == 0


@fake_pointers
def test_swiglu_ffn_backward(nv):
    def call(dh=A, x=A, ldx=64, wg=A, wu=A, ldw=64, g=A, u=A, m=4, n=8, k=64, dx=A, dwg=A, dwu=A, ws=A, wsb=1 << 40):
        return nv.nvfp4_swiglu_ffn_backward(dh, x, ldx, wg, wu, ldw, g, u, m, n, k, dx, dwg, dwu, ws, wsb, None)

    assert call(dh=None) == call(x=None) == call(wg=None) == call(wu=None) == call(g=None) == call(u=None) == -1
    assert call(dwg=None) == call(dwu=None) == call(dx=None, dwg=None, dwu=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-1) == call(ldx=63) == call(ldw=63) == -2
    for name in ("dh", "x", "wg", "wu", "g", "u", "dx", "dwg", "dwu"):
        assert call(**{name: OFF8}) == -7, name
    need = nv.nvfp4_swiglu_ffn_backward_workspace_bytes(4, 8, 64, 64, 64)
    assert need >= 4 * 2 * 64 * 2
    assert call(ws=None) == call(wsb=need - 1) == -6
    assert call(ws=P(0x100010)) == -7
    assert call(m=0, n=0) == 0


def test_wrappers_refuse_host_tensors(nv):
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    q, sc, S = torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 4), dtype=torch.uint8), torch.ones(1)
    for call in (lambda: nv.mx_quantize(x), lambda: nv.mx_dequant(q, sc[:, :2].contiguous()),
                 lambda: nv.matmul(x, q, sc, S), lambda: nv.matmul_grad_input(x, q, sc, S),
                 lambda: nv.mx_matmul((q, sc[:, :2].contiguous()), (q, sc[:, :2].contiguous())),
                 lambda: nv.swiglu_ffn(x, x, x), lambda: nv.swiglu_ffn_backward(x, x, x, x, x, x)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_wrappers_refuse(nv):
    """Shapes, types and layouts that the calls do not take, on real tensors."""
    dev = torch.device("cuda:0")

    def z(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device=dev)

    u8 = torch.uint8
    x, q, sc, S = z(4, 64), z(8, 32, dtype=u8), z(8, 4, dtype=u8), z(1, dtype=torch.float32)
    a, b = (z(4, 32, dtype=u8), z(4, 2, dtype=u8)), (z(8, 32, dtype=u8), z(8, 2, dtype=u8))
    ok = z(4, 8)
    cases = [
        (ValueError, lambda: nv.mx_quantize(x[:, ::2])), (ValueError, lambda: nv.mx_quantize(x[0])),
        (TypeError, lambda: nv.mx_quantize(x.half())), (ValueError, lambda: nv.mx_dequant(a[0], b[1])),
        (ValueError, lambda: nv.mx_dequant(*a, cols=32)), (TypeError, lambda: nv.mx_dequant(*a, out_dtype=torch.float16)),
        (ValueError, lambda: nv.mx_matmul(a, (z(8, 16, dtype=u8), z(8, 1, dtype=u8)))),
        (ValueError, lambda: nv.mx_matmul(a, b, out=z(8, 4))), (ValueError, lambda: nv.mx_matmul(a, (b[0], S))),
        (ValueError, lambda: nv.mx_matmul_grad_input(x, *b)), (ValueError, lambda: nv.mx_matmul_grad_input(ok, *b, cols=65)),
        (TypeError, lambda: nv.matmul(x.float(), q, sc, S)), (ValueError, lambda: nv.matmul(x[:, :32], q, sc, S)),
        (ValueError, lambda: nv.matmul(x.t(), q, sc, S)), (ValueError, lambda: nv.matmul(x, q, sc[:, :3].contiguous(), S)),
        (ValueError, lambda: nv.matmul(x, q, sc, S.double())), (ValueError, lambda: nv.matmul(x, q, sc, S, out=ok.float())),
        (nv.NVFP4Error, lambda: nv.matmul(x, q, sc, S, block=0)), (TypeError, lambda: nv.matmul(x, q, sc, S, out_dtype=u8)),
        (ValueError, lambda: nv.matmul(x[:1].expand(4, 64), q, sc, S)),
        (ValueError, lambda: nv.matmul_grad_input(x, q, sc, S)),
        (ValueError, lambda: nv.swiglu_ffn(x, z(8, 32), z(8, 32))), (ValueError, lambda: nv.swiglu_ffn(x, z(8, 64), z(9, 64))),
        (ValueError, lambda: nv.swiglu_ffn(x, z(8, 64), z(8, 72)[:, :64])),
        (ValueError, lambda: nv.swiglu_ffn_backward(ok, x, z(8, 64), z(8, 64), ok, z(4, 9))),
        (nv.NVFP4Error, lambda: nv.swiglu_ffn(z(4, 72)[:, 2:66], z(8, 64), z(8, 64))),
        (nv.NVFP4Error, lambda: nv.swiglu_ffn_backward(ok, x, z(8, 64), z(8, 64), ok, ok, ws=z(8))),
    ]
    for i, (error, call) in enumerate(cases):
        with pytest.raises(error):
            call()
            pytest.fail(f"case {i} passed")
