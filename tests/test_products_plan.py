"""The sizes that the products are compared at reach every form that the library's rule can choose, so that a changed rule
cannot leave one untested."""
import math
import random
import subprocess
from pathlib import Path

import pytest

import product_shapes

HERE = Path(__file__).resolve().parent


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "product_plan_of"
    subprocess.run(["g++", "-O2", "-std=c++17", f"-I{HERE.parent / 'paper_2606_07618_amd' / 'csrc'}", "-o", str(exe),
                    str(HERE / "product_plan_of.cpp")], check=True)

    def ask(op, shapes):
        text = "\n".join(f"{op} {m} {n} {k}" for m, n, k in shapes)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(shapes)
        return out
    return ask


@pytest.mark.parametrize("op", list(product_shapes.SHAPES))
def test_every_form_is_compared(forms, op):
    rng = random.Random(11)

    def size(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    unit = 16 if op in ("linear", "grad") else 1
    grid = [(size(1, 20000), size(1, 40000), max(1, size(16, 40000) // unit) * unit) for _ in range(100000)]
    reached, tested = set(forms(op, grid)), set(forms(op, product_shapes.SHAPES[op]))
    assert reached - tested <= {"dot"}, reached - tested      # one to four rows have sizes of their own


def test_long_products_go_around(forms):
    shapes = [s[:3] for s in product_shapes.LONG]
    assert all(form.startswith("stream") for form in forms("linear", shapes))
    assert all(int(t) >= 3 for t in forms("turns", shapes))


@pytest.mark.parametrize("k", [64, 1024, 14336])
def test_estimates_grow_with_the_workgroups(forms, k):
    """One more tile never makes a product faster: the estimates do not fall anywhere, full chip and more among them."""
    rows = [list(map(float, line.split())) for line in forms("times", [(w, 64, k) for w in range(1, 600)])]
    for lo, hi in zip(rows, rows[1:]):
        assert all(b >= a for a, b in zip(lo, hi)), (lo, hi)
