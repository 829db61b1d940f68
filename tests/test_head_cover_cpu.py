"""The sizes of the device tests reach every kernel that the plan of the output head can choose:
asked of the plan itself, so that a change of its estimates shows here."""
import os
import subprocess

import pytest

from head_sizes import SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def seen(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cover") / "head_cover_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror",
                    "-I", os.path.join(ROOT, "paper_2606_13894_amd", "csrc"),
                    os.path.join(ROOT, "tests", "head_cover_check.cpp"), "-o", exe], check=True)
    args = [str(n) for size in SIZES for n in size]
    out = subprocess.run([exe, *args], capture_output=True, text=True, check=True).stdout
    return [line.split() for line in out.splitlines()]


def test_products_are_covered(seen):
    """Each tile, with one, two, three and more stages; split and unsplit sums."""
    got = {(v[0], int(v[1]), min(int(v[2]), 2), min(int(v[3]), 3)) for v in seen if len(v) == 4}
    want = set()
    for tile in (64, 128, 256):
        for kind in ("scores", "gradients1", "dx1", "dweight2"):
            want |= {(kind, tile, 1, s) for s in (1, 2, 3)}
        # gradients in one number are for more than 256 tokens, more than four stages
        want |= {("dx1", tile, 2, 3), ("dx2", tile, 2, 3), ("dweight1", tile, 1, 3),
                 ("dweight1", tile, 2, 3)}
    want |= {(kind, 64, 1, s) for kind in ("gradients2", "dx2") for s in (1, 2, 3)}
    want.add(("gradients2", 128, 1, 3))
    assert want <= got, sorted(want - got)


def test_few_tokens_and_ranges_are_covered(seen):
    few = {(int(v[1]), int(v[2])) for v in seen if v[0] == "few"}
    assert few == {(rows, waves) for rows in (8, 16) for waves in (1, 4, 8, 16)}
    assert {min(int(v[1]), 2) for v in seen if v[0] == "ranges"} == {1, 2}
