"""That the sizes of shape_sizes.py take every kind of tile, by the header that the library chooses with, compiled for the host: a new table of paces
that leaves a tile untested fails here.  No GPU is involved."""
import os
import subprocess

import pytest

from shape_sizes import I8, ORTH

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("shapes") / "shapes_check")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I", os.path.join(ROOT, "paper_2402_01798_amd", "csrc"), os.path.join(ROOT, "tests", "shapes_check.cpp"), "-o", exe])
    return lambda lines: subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True).stdout.splitlines()


def test_8_bit_products(ask):
    assert sorted(I8) == sorted(["64", "128", "192", "256", "192x256", "128x320", "256x128", "128x256"])
    for name, sizes in I8.items():
        assert [a.split()[0] for a in ask(["i8 %d %d %d" % s for s in sizes])] == [name] * len(sizes)
        assert name == "128x256" or any(m % 64 and n % 64 and k % 128 for m, n, k in sizes)


@pytest.mark.parametrize("precision", sorted(ORTH))
def test_orthogonalised_matrices(ask, precision):
    """Every tile for each of a step's products, the two symmetric ones and the last; of the last, both ways round."""
    pairs = int(precision == "split")
    every = {"64", "128", "128 alone", "192", "256"}
    symmetric = ask(["orth %d %d %d %d 1 %d" % (pairs, r, r, c, n) for r, c, n in ORTH[precision]])
    squared = ask(["orth %d %d %d %d 1 %d" % (pairs, r, r, r, n) for r, c, n in ORTH[precision]])
    applied = ask(["orth %d %d %d %d 0 %d" % (pairs, r, c, r, n) for r, c, n in ORTH[precision]])
    turned = ask(["orth %d %d %d %d 0 %d" % (pairs, c, r, r, n) for r, c, n in ORTH[precision]])
    assert set(symmetric) == set(squared) == set(applied) == set(turned) == every


def test_what_larger_products_take(ask):
    """Sizes of layers."""
    got = ask(["i8 8192 8192 8192", "i8 1037 8192 4096", "i8 5000 5000 3000", "i8 24 14336 4096", "i8 64 64 65536", "i8 100 4096 4096"])
    assert [g.split()[0] for g in got] == ["256", "128x320", "192", "few", "64", "64"]
    assert int(got[4].split()[1]) > 1 and got[5].split()[1] == "1"
    assert ask(["orth 0 4096 4096 4096 1 1", "orth 0 4096 4096 4096 0 1", "orth 1 1024 1024 4096 1 4", "orth 1 1024 4096 1024 0 4"]) == ["192", "256", "64", "256"]
