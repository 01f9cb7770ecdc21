"""The sizes that products of 8-bit integers and of grouped rows are compared at reach every form that the library's rule can
choose, so that a changed rule cannot leave one untested."""
import math
import random
import subprocess
from pathlib import Path

import pytest

import int8_grouped_shapes as shapes

HERE = Path(__file__).resolve().parent


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "int8_grouped_plan_of"
    subprocess.run(["g++", "-O2", "-std=c++17", f"-I{HERE.parent / 'paper_2606_07618_amd' / 'csrc'}", "-o", str(exe),
                    str(HERE / "int8_grouped_plan_of.cpp")], check=True)

    def ask(op, sizes):
        text = "\n".join(f"{op} {a} {b} {c}" for a, b, c in sizes)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(sizes)
        return out
    return ask


def spread(count, *ranges):
    rng = random.Random(13)
    return [tuple(int(math.exp(rng.uniform(math.log(lo), math.log(hi)))) for lo, hi in ranges) for _ in range(count)]


def test_every_form_of_the_8_bit_product(forms):
    grid = spread(100000, (1, 20000), (1, 40000), (16, 40000))
    grid += [(m, -(-n // 8) * 8, k) for m, n, k in grid]
    reached, tested = set(forms("int8", grid)), forms("int8", shapes.INT8)
    assert reached - set(tested) <= {"dot"}, reached - set(tested)        # one to four rows have tests of their own


def grouped(sizes, outer):
    return sum(sizes), len(sizes), outer


def test_every_form_of_the_grouped_products(forms):
    grid = spread(100000, (1, 40000), (1, 300), (16, 40000))
    few = set(forms("grouped", [grouped(sizes, n) for sizes, n in shapes.FEW]))
    tall = set(forms("grouped", [grouped(shapes.TALL, shapes.TALL_OUTER)]))
    tall_turned = set(forms("turned", [grouped(shapes.TALL, shapes.TALL_OUTER)]))
    small = {"128 x 128 by 256"}                          # has tests of its own
    assert set(forms("grouped", grid)) == few | tall | small
    assert set(forms("turned", grid)) == tall_turned | small
    assert {"16 x 64 by 512", "16 x 128 by 256", "32 x 64 by 256", "32 x 128 by 256"} == few
    assert tall == tall_turned == {"256 x 256 by 512"}
