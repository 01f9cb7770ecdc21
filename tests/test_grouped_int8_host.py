"""Refusals of the grouped and the 8-bit products' C entry points and wrappers, on the host: validation returns before any
launch.  Made-up device addresses only where no GPU is visible."""
import ctypes
import re
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parents[1]
P = ctypes.c_void_p
A = P(0x100000)                       # never dereferenced
OFF8, OFF2, OFF1 = P(0x100008), P(0x100002), P(0x100001)
BIG = 1 << 62

fake_pointers = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                   reason="made-up device addresses only where no GPU is visible")


@pytest.fixture(scope="module")
def nv():
    import paper_2606_07618_amd as nv
    return nv


def test_every_declared_symbol_is_exported_and_bound(nv):
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "nvfp4ss.h").read_text(), flags=re.S)
    names = set(re.findall(r"\b(int8_\w+|nvfp4_grouped\w*)\s*\(", text))
    assert len(names) == 8
    for n in names:
        assert getattr(nv.lib, n).argtypes is not None, n


@fake_pointers
@pytest.mark.parametrize("grad", [False, True])
def test_grouped(nv, grad):
    def call(x=A, ld=64, offsets=A, q=A, sc=A, block=16, S=A, rows=4, experts=3, n=64, k=64, dtype=1, clear=1, out=A, ws=A,
             wsb=1 << 40):
        if grad:
            return nv.nvfp4_grouped_product_grad_input(x, ld, offsets, q, sc, block, S, rows, experts, n, k, dtype, clear, out,
                                                       ws, wsb, None)
        return nv.nvfp4_grouped_product(x, ld, offsets, q, sc, block, S, rows, experts, n, k, dtype, clear, out, None)

    assert call(x=None) == call(offsets=None) == call(q=None) == call(sc=None) == call(S=None) == call(out=None) == -1
    assert call(experts=0, offsets=None) == -1
    assert call(rows=-1) == call(experts=-1) == call(n=-1) == call(k=-64) == call(k=72) == call(ld=56) == -2
    assert call(rows=1 << 31) == call(rows=BIG) == call(experts=(1 << 20) + 1) == call(experts=BIG) == call(ld=1 << 22) == -2
    assert call(n=(1 << 20) + 16, ld=1 << 21) == call(k=1 << 21, ld=1 << 21) == -2
    # more workgroups than one launch holds
    assert call(rows=(1 << 31) - 1, n=1 << 20, k=1 << 20, ld=1 << 20) == -2
    assert call(block=24) == call(block=0) == -3
    assert call(dtype=2) == call(dtype=-1) == -4
    assert call(x=OFF8) == call(q=OFF8) == call(out=OFF8) == call(S=OFF2) == call(offsets=OFF2) == -7
    assert call(rows=0, x=None) == call(**{"k" if grad else "n": 0}, out=None) == call(experts=0, clear=0, out=None) == 0
    if not grad:
        assert call(ld=68) == -7
        return
    need = nv.nvfp4_grouped_product_grad_input_workspace_bytes(200, 510, 510)
    assert need >= 200 * 512 * 2                       # rows of 510 values are copied to rows of 512
    assert nv.nvfp4_grouped_product_grad_input_workspace_bytes(200, 512, 512) == 0
    big = dict(rows=200, n=510, ld=510)
    assert call(ws=None, **big) == call(wsb=need - 1, **big) == -6
    assert call(ws=P(0x100010), **big) == -7
    assert nv.nvfp4_grouped_product_grad_input_workspace_bytes(8, -1, 64) == -2


@fake_pointers
def test_int8_quant(nv):
    def call(x=A, dtype=1, rows=4, cols=70, ldx=70, q=A, sc=A):
        return nv.int8_quant(x, dtype, rows, cols, ldx, q, sc, None)

    assert call(x=None) == call(q=None) == call(sc=None) == -1
    assert call(rows=-1) == call(cols=-1) == call(rows=BIG) == call(ldx=69) == call(ldx=1 << 22) == -2
    assert call(cols=1 << 17, ldx=1 << 17) == -2
    assert call(dtype=2) == -4
    assert call(x=OFF1) == call(x=OFF2, dtype=0) == call(q=OFF8) == call(sc=OFF2) == -7
    assert call(rows=0, x=None) == 0


@fake_pointers
def test_int8_matmul(nv):
    def call(aq=A, asc=A, bq=A, bsc=A, m=4, n=8, k=60, dtype=1, out=A, ws=A, wsb=1 << 40):
        return nv.int8_product(aq, asc, bq, bsc, m, n, k, dtype, out, ws, wsb, None)

    assert call(aq=None) == call(asc=None) == call(bq=None) == call(bsc=None) == call(out=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-1) == call(n=1 << 21) == call(k=(1 << 17) - 15) == call(m=BIG) == -2
    assert call(dtype=-1) == -4
    assert call(aq=OFF8) == call(bq=OFF8) == call(out=OFF8) == call(asc=OFF2) == call(bsc=OFF2) == -7
    need = nv.int8_product_workspace_bytes(200, 80, 9600)
    assert need > 0
    big = dict(m=200, n=80, k=9600)
    assert call(ws=None, **big) == call(wsb=need - 1, **big) == -6
    assert call(ws=P(0x100010), **big) == -7
    assert call(m=0, aq=None) == call(n=0, out=None) == 0
    assert nv.int8_product_workspace_bytes(1, 1, 1 << 17) == -2


@fake_pointers
def test_int8_grad_input(nv):
    def call(dy=A, ld=40, q=A, sc=A, m=4, n=40, k=60, dtype=1, out=A, ws=A, wsb=1 << 40):
        return nv.int8_product_grad_input(dy, ld, q, sc, m, n, k, dtype, out, ws, wsb, None)

    size = nv.int8_product_grad_input_workspace_bytes
    assert call(dy=None) == call(q=None) == call(sc=None) == call(out=None) == -1
    assert call(m=-1) == call(n=-1) == call(k=-1) == call(ld=39) == call(ld=1 << 22) == call(k=1 << 17) == -2
    assert call(dtype=2) == -4
    assert call(dy=OFF8) == call(q=OFF8) == call(out=OFF8) == call(sc=OFF2) == -7
    need = size(200, 510, 500, 510)
    assert need >= 200 * 512 * 2 + 512 * 512 * 2
    big = dict(m=200, n=510, k=500, ld=510)
    assert call(ws=None, **big) == call(wsb=need - 1, **big) == -6
    assert call(ws=P(0x100010), **big) == -7
    assert call(m=0, dy=None) == call(k=0, out=None) == 0
    assert size(8, -1, 64, 64) == -2


@pytest.mark.gpu
def test_wrappers_refuse(nv):
    dev = torch.device("cuda:0")

    def z(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device=dev)

    u8, i8, i32, f32 = torch.uint8, torch.int8, torch.int32, torch.float32
    x, off, w = z(4, 64), z(4, dtype=i32), (z(3, 8, 32, dtype=u8), z(3, 8, 4, dtype=u8), z(3, dtype=f32))
    assert nv.grouped_matmul(x, off, *w).shape == (4, 8)
    for bad in (dict(x=x.cpu()), dict(x=z(4, 80)), dict(x=z(4)), dict(x=z(64, 4).t()), dict(offsets=z(3, dtype=i32)),
                dict(offsets=z(4, dtype=torch.int64)), dict(offsets=off.cpu()), dict(q=w[0][0]), dict(q=w[0].transpose(0, 1)),
                dict(scales=z(3, 8, 2, dtype=u8)), dict(scales=z(96, dtype=u8)), dict(S=z(1, dtype=f32)),
                dict(S=z(3)), dict(out=z(4, 9)), dict(out=z(4, 8, dtype=f32))):
        args = dict(x=x, offsets=off, q=w[0], scales=w[1], S=w[2], **({"out": bad["out"]} if "out" in bad else {}))
        with pytest.raises(ValueError):
            nv.grouped_matmul(**{**args, **bad})
    with pytest.raises(TypeError):
        nv.grouped_matmul(x.float(), off, *w)
    with pytest.raises(TypeError):
        nv.grouped_matmul(x, off, *w, out_dtype=torch.float16)
    with pytest.raises(nv.NVFP4Error):
        nv.grouped_matmul(x, off, *w, block=0)
    with pytest.raises(ValueError):
        nv.grouped_matmul_grad_input(z(4, 9), off, *w)
    with pytest.raises(ValueError):
        nv.grouped_matmul_grad_input(z(4, 7), off, z(3, 7, 32, dtype=u8), z(3, 7, 4, dtype=u8), w[2], ws=z(1, dtype=u8).cpu())
    with pytest.raises(nv.NVFP4Error):
        nv.grouped_matmul_grad_input(z(4, 7), off, z(3, 7, 32, dtype=u8), z(3, 7, 4, dtype=u8), w[2], ws=z(1, dtype=u8))

    a, b = (z(4, 64, dtype=i8), z(4, dtype=f32)), (z(8, 64, dtype=i8), z(8, dtype=f32))
    assert nv.int8_matmul(a, b).shape == (4, 8)
    for bad in ((z(4, 60, dtype=i8), a[1]), (z(4, 80, dtype=i8), a[1]), (a[0], z(5, dtype=f32)), (a[0], z(4)), (a[0].cpu(), a[1]),
                (z(4, 64, dtype=u8), a[1]), (z(64, 4, dtype=i8).t(), a[1]), (z(64, dtype=i8), a[1])):
        with pytest.raises(ValueError):
            nv.int8_matmul(bad, b)
    with pytest.raises(TypeError):
        nv.int8_matmul(a, b, out_dtype=torch.int32)
    for bad in (z(4), x.cpu(), z(64, 4).t()):
        with pytest.raises(ValueError):
            nv.int8_quantize(bad)
    for bad in (x.half(), x.double(), z(4, 4, dtype=i8)):
        with pytest.raises(TypeError):
            nv.int8_quantize(bad)
    with pytest.raises(ValueError):
        nv.int8_quantize(z(4, 60), out=(z(4, 60, dtype=i8), z(4, dtype=f32)))
    with pytest.raises(ValueError):
        nv.int8_matmul_grad_input(z(4, 9), *b)
    for cols in (48, 65, 0, -1):
        with pytest.raises(ValueError):
            nv.int8_matmul_grad_input(z(4, 8), *b, cols=cols)
    assert nv.int8_matmul_grad_input(z(4, 8), *b, cols=49).shape == (4, 49)
