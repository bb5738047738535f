"""Host-only: what a piece of the classes takes of a loss's workspace, and where things lie in it."""
import math
import os
import random
import shutil
import subprocess

import pytest

from paper_1810_09868_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("pieces") / "pieces_check")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-o", exe, os.path.join(ROOT, "tests", "host", "pieces_check.cpp")])

    def of(shapes):
        text = "\n".join("%d %d %d %d" % s for s in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        assert len(out) == len(shapes)
        return [tuple(int(v) for v in line.split()) for line in out]

    return of


def test_a_piece_takes_what_it_says(ask):
    rng = random.Random(11)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    shapes = [(d, n, i, k) for d in (B.F32, B.BF16) for n in (1, 64, 65, 256, 512, 513, 8192) for i in (64, 100, 2048) for k in (1 << 17, 1 << 20, (1 << 21) + 5, 1 << 24)]
    shapes += [(rng.randrange(2), log(1, 1 << 22), log(1, 1 << 20), log(1, 1 << 24)) for _ in range(2000)]
    for s, (takes, may, follow, _) in zip(shapes, ask(shapes)):
        assert takes <= may and follow, (s, takes, may, follow)


def test_shapes_of_the_gpu_tests_have_two_pieces(ask):
    assert [line[3] for line in ask([(B.BF16, 512, 64, 300001), (B.BF16, 449, 33, 270000)])] == [2, 2]


def test_workspaces_of_few_rows_stay_near_a_piece():
    # bf16 rows up to 512 keep what rounding leaves of dz beside it.  Beyond the piece: parts of da, up to 256 tiles of 256 x 256 fp32 numbers and as
    # many again where the last round of them is full (128 MB); activations and the like (16 MB)
    for n, i, k in ((512, 2048, 1 << 20), (256, 64, 1 << 21), (512, 64, 1 << 24)):
        assert B.vgg_fc_xent_bwd_workspace_bytes(B.BF16, n, i, k) < (512 + 128 + 16) << 20
