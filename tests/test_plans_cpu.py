"""Host-only: the shapes that the GPU tests take for every kernel variant do go there, by the library's own rules."""
import math
import os
import random
import shutil
import subprocess

import pytest

from paper_1810_09868_amd import binding as B

from plan_shapes import MUON_256, W4_TILES, XENT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plans") / "plans_check")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-o", exe, os.path.join(ROOT, "tests", "host", "plans_check.cpp")])
    return lambda lines: subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()


def test_shapes_reach_their_variants(ask):
    def muon(shapes):
        return ask(["muon %d %d %d" % (b, min(m, n), max(m, n)) for b, m, n in shapes])

    assert muon(MUON_256) == ["256"] * len(MUON_256)
    assert muon([(1, 4096, 25088), (1, 25088, 4096), (7, 512, 4608), (1, 1000, 4096)]) == ["256", "256", "128", "128"]
    assert ask(["w4 %d %d %d %d" % k for k in W4_TILES]) == ["%d %d" % v for v in W4_TILES.values()]
    for dtype in (B.F32, B.BF16):
        assert {v for k, v in W4_TILES.items() if k[0] == dtype} == {(nt, rt) for nt in (1, 2, 4) for rt in (1, 2, 4)}
    # the network's dense layers, batch 1, 10 and 100
    assert ask(["w4 1 1 25088 4096", "w4 1 10 4096 4096", "w4 1 100 25088 4096", "w4 1 100 4096 4096", "w4 0 100 4096 1000"]) == [
        "row", "tile", "4 4", "4 2", "4 2"]


def test_matrices_of_few_rows_that_are_too_long_go_by_tiles(ask):
    # (a launch a step reads the square of its workgroups: no more of them than run at once)
    shapes = [(2, 1, 1), (2, 64, 448), (1, 640, 64), (2, 64, 98304), (1, 131072, 64), (2, 64, 131072), (1, 64, 196608), (2, 1000000, 16), (1, 1, 1 << 22), (2, 65, 65)]
    assert ask(["few %d %d %d" % s for s in shapes]) == ["1"] * 5 + ["0"] * 5


def test_losses_over_many_classes_reach_their_variants(ask):
    assert ask(["xent %d %d %d %d" % k for k in XENT]) == list(XENT.values())
    # every width of tile, for every product, in either type
    for dtype in (B.F32, B.BF16):
        for product in range(4):
            seen = {v.split()[2 + product] for k, v in XENT.items() if k[0] == dtype and v != "small"}
            assert seen == ({"64", "128"} if product == 1 and dtype == B.F32 else {"64", "128", "256"}), (dtype, product, seen)


def test_plans_of_losses_hold_together(ask):
    rng = random.Random(5)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    shapes = [(rng.randrange(2), log(1, 1 << 22), log(1, 1 << 20), log(1, 1 << 24)) for _ in range(3000)]
    shapes += [(d, n, i, k) for d in (0, 1) for n in (1, 64, 65, 1 << 22) for i in (1, 64, 1 << 20) for k in (1, 256, 257, 1 << 24)]
    assert [ask(["xent %d %d %d %d" % s])[0].split()[0] for s in ((1, 8200, 64, 40000), (0, 16390, 70, 20011), (1, 30000, 130, 9000))] == ["2", "3", "2"]
    out = ask(["xent %d %d %d %d" % s for s in shapes])
    assert len(out) == len(shapes)
    for s, line in zip(shapes, out):
        assert line == "small" or line[0].isdigit(), (s, line)
