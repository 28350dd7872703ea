"""Which kernel a product takes, and in how many pieces, asked of the library's own estimate on the host: the shapes with which the
GPU tests reach every kernel, alone, two in a launch and in pieces, still do."""
import os
import shutil
import subprocess

import pytest

import layer_shapes as S
from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
PKG = os.path.join(ROOT, "paper_1610_02132_amd")
LIB = os.path.join(PKG, "libqsgd.so")
pytestmark = pytest.mark.skipif(not shutil.which(HIPCC) or not os.path.exists(LIB), reason="needs hipcc and the library")

ASK = r"""
#include "qsgd_layer.hip"
#include <cstdio>
int main() {   // M N K -> kernel, pieces
  unsigned M, N, K;
  while (std::scanf("%u %u %u", &M, &N, &K) == 3) {
    const ProductPlan p = product_plan(M, N, K);
    std::printf("%u %u\n", p.kind, p.splits);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    path = tmp_path_factory.mktemp("ask")
    (path / "ask.hip").write_text(ASK)
    subprocess.run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O1", "-Wno-unused-function",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), str(path / "ask.hip"),
                    "-o", str(path / "ask"), "-L", PKG, "-lqsgd", "-Wl,-rpath," + PKG], check=True, capture_output=True)

    def answers(rows):
        text = "".join(" ".join(map(str, r)) + "\n" for r in rows)
        out = subprocess.run([str(path / "ask")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return answers


def test_products_in_pieces(plan):
    assert dict(zip(S.IN_PIECES, plan(S.IN_PIECES))) == S.IN_PIECES
    kinds = {kind for kind, _ in S.IN_PIECES.values()}
    assert kinds == {S.FEW, S.TILE64_DEEP, S.TILE128, S.TILE128X64, S.TILE256}
    for kind in kinds:   # joined four to a thread, and one
        assert {N % 4 == 0 for (_, N, _), (k, _) in S.IN_PIECES.items() if k == kind} == {True, False}


def test_kernels_that_no_product_takes_in_pieces(plan):
    """(The tiles of 64 with two stages, and little depth: no test of theirs in pieces is missing.)"""
    rows = [(M, N, K) for M in (1, 33, 64, 200, 700, 2000, 9000) for N in (1, 60, 64, 130, 500, 2000, 9000)
            for K in (4097, 5000, 9000, 20_000, 60_000, 130_816, 130_817, 400_000)]
    assert {kind for kind, pieces in plan(rows) if pieces > 1} <= {kind for kind, _ in S.IN_PIECES.values()}


def both(plan, shapes):
    dx, dw = plan([(M, K, N) for M, N, K in shapes]), plan([(N, K, M) for M, N, K in shapes])
    return dict(zip(shapes, zip(dx, dw)))


def test_gradients_in_one_launch(plan):
    assert both(plan, S.PAIRS) == {s: ((a, 1), (b, 1)) for s, (a, b) in S.PAIRS.items()}
    assert {a for a, _ in S.PAIRS.values()} == {S.TILE64_DEEP, S.TILE64, S.TILE128, S.TILE128X64, S.TILE256, S.SHALLOW}


def test_gradients_in_pieces(plan):
    assert both(plan, S.BACKWARD_IN_PIECES) == S.BACKWARD_IN_PIECES
