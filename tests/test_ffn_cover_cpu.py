"""The sizes of the device tests reach every kernel that the plan of the block's products can
choose: asked of the plan itself, so that a change of its estimates shows here."""
import os
import subprocess

import pytest

from ffn_sizes import FEW, TILES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cover") / "ffn_cover_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror",
                    "-I", os.path.join(ROOT, "paper_2606_13894_amd", "csrc"),
                    os.path.join(ROOT, "tests", "ffn_cover_check.cpp"), "-o", exe], check=True)
    args = [str(n) for size in TILES + FEW for n in size]
    out = subprocess.run([exe, *args], capture_output=True, text=True, check=True).stdout
    return [line.split() for line in out.splitlines()]


def test_tiles_are_covered(lines):
    seen = {(kind, int(tile), min(int(splits), 2), min(int(stages), 4))
            for kind, tile, splits, stages in (v for v in lines if len(v) == 4)}
    want = set()
    for tile in (128, 256):
        for kind in ("gate_up", "down", "gate_grad", "dx", "dw"):
            # the plan gives the gate's gradients the largest tile at long sums only
            stages = (4,) if (kind, tile) == ("gate_grad", 256) else (1, 2, 3, 4)
            want |= {(kind, tile, 1, s) for s in stages}
            if kind in ("down", "dx", "dw"):
                want.add((kind, tile, 2, 4))
    assert want <= seen, sorted(want - seen)
    # an even and an odd number of parts, so that dx is also cut inside its two segments
    for kind in ("down", "dx", "dw"):
        parts = {(int(t), int(s) % 2) for k, t, s, _ in (v for v in lines if len(v) == 4)
                 if k == kind and int(s) > 1}
        assert parts >= {(128, 0), (128, 1), (256, 0), (256, 1)}, (kind, parts)


def test_few_tokens_are_covered(lines):
    seen = {tuple(v) for v in lines if len(v) == 3}
    want = {(kind, rows, waves) for kind in ("few_gate_up", "few_down") for rows in ("8", "16")
            for waves in ("4", "8", "16")}
    assert want == seen, (sorted(want - seen), sorted(seen - want))
