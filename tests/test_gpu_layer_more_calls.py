"""Backward passes of long rows captured into graphs and on another stream; long rows and every kind of tile with folded grids."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2402_01798_amd import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def rows(cols, seed, n=9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, cols, generator=g, device="cuda") + 5000.0
    return x, torch.randn(n, cols, generator=g, device="cuda")


def buffers(x):
    n, cols = x.shape
    return {"y": torch.empty_like(x), "stats": torch.empty(n, 2, device="cuda"), "dx": torch.empty_like(x), "dw": torch.empty(cols, device="cuda"),
            "db": torch.empty(cols, device="cuda"), "dw2": torch.empty(cols, device="cuda"), "dy2": torch.empty_like(x),
            "ws": torch.empty(B.layernorm_workspace_bytes(n, cols), dtype=torch.uint8, device="cuda").fill_(255)}


def passes(x, dy, b):
    """dx apart from what it is made of, sums alone, dx in place."""
    B.tq_layernorm_forward(x, None, None, b["y"], b["stats"])
    B.tq_layernorm_backward(x, dy, None, b["stats"], b["dx"], b["dw"], b["db"], b["ws"])
    B.tq_layernorm_backward(x, dy, None, b["stats"], None, b["dw2"], None, b["ws"])
    b["dy2"].copy_(dy)
    B.tq_layernorm_backward(x, b["dy2"], None, b["stats"], b["dy2"], b["dw2"], None, b["ws"], accumulate=True)
    return [b[k] for k in ("y", "dx", "dw", "db", "dw2", "dy2")]


@pytest.mark.parametrize("cols", [900, 17003, 33001])
def test_captured_and_replayed(cols):
    x, dy = rows(cols, 1)
    b = buffers(x)
    passes(x, dy, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes(x, dy, b)
    for seed in (2, 3, 4):
        for t, new in zip((x, dy), rows(cols, seed)):
            t.copy_(new)
        graph.replay()
        replayed = [t.clone() for t in got]
        torch.cuda.synchronize()
        want = passes(*rows(cols, seed), buffers(x))
        assert all(torch.equal(a, w) for a, w in zip(replayed, want))
        assert torch.equal(want[4], 2 * want[2]) and torch.equal(want[5], want[1])


@pytest.mark.parametrize("cols", [900, 17003, 33001])
def test_on_another_stream(cols):
    x, dy = rows(cols, 5)
    want = [t.clone() for t in passes(x, dy, buffers(x))]
    b = buffers(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = passes(x, dy, b)
    side.synchronize()
    assert all(torch.equal(a, w) for a, w in zip(got, want))


def test_with_a_folded_grid():
    from paper_2402_01798_amd import build
    assert os.path.exists(build.FOLD_TEST_LIB), "build it first: python -m paper_2402_01798_amd.build"
    env = dict(os.environ, TQ_TEST_MAX_GRID_X="16", TQ_LIBRARY_PATH=build.FOLD_TEST_LIB)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_norm_rows.py::test_some_of_the_gradients_and_in_place",
           "tests/test_gpu_norm_rows.py::test_a_mean_far_above_the_deviations", "tests/test_gpu_i8_tiles.py", "tests/test_gpu_orth_errors.py::test_updates"]
    r = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
