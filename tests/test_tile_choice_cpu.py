"""The lists of tests/test_gpu_operator_tiles.py reach every tile that the host
may choose: its own rules (csrc/ops/cost.h), compiled for the host."""

import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")
from tests.test_gpu_operator_tiles import APPLY, ORTHO, PARTS, PRODUCT  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OPS = os.path.join(ROOT, "paper_2608_28941_amd", "csrc", "ops")


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    """choose(lines): the numbers that the rules give for each line."""
    cxx = shutil.which("g++") or shutil.which("clang++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("tiles") / "choice")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-I", OPS, os.path.join(ROOT, "tests", "host_tile_choice.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, timeout=60, check=True)
        got = [tuple(map(int, x.split())) for x in out.stdout.splitlines()]
        assert len(got) == len(lines)
        return got

    return ask


def test_orthogonalised_steps(choose):
    """32, 64, 128 (with either ring), 192 and 256, for the Gram product, whole and
    split, for the products of the short side and for those with X."""
    gram, parts, short, long = set(), set(), set(), set()
    for tile, splits, deep, q, q_deep, x, x_deep in choose([f"ortho {s} {l} {b}" for b, s, l in ORTHO]):
        (parts if splits > 1 else gram).add((tile, deep if tile == 2 else None))
        short.add((q, q_deep if q == 2 else None))
        long.add((x, x_deep if x == 2 else None))
    every = {(0, None), (1, None), (2, 1), (2, 0), (3, None), (4, None)}
    assert gram == every and parts == every and short == every and long == every


@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("name", list(APPLY))
def test_a_4_bit_matrix_times_real_columns(choose, name, trans):
    cases = [c for c in APPLY[name] if c[0] == trans]
    got = choose([f"apply {t} {k} {m} {n} {PARTS[name]}" for t, k, m, n in cases])
    assert {tile for tile, _ in got} == {0, 1, 2, 3, 4}
    assert {splits > 1 for _, splits in got} == {False, True}


def test_two_4_bit_matrices(choose):
    assert {t for t, in choose([f"product {M} {N} {k}" for M, N, k in PRODUCT])} == {0, 1, 2, 3}
