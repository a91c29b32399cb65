"""examples/engine_batches.py: the scheduler's batches executed over a paged cache, timed, fitted and estimated with."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    import __graft_entry__
    __graft_entry__.build()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("engine_batches", os.path.join(ROOT, "examples", "engine_batches.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
def test_the_example_runs(ex, fmt):
    coef, mape, ttft, executed, off = ex.main(["--layers", "2", "--prompts", "40", "--seqs", "16", "--format", fmt])
    assert np.isfinite(coef).all() and np.isfinite(mape)
    # the estimate is of the batches that were executed: the same number of them, by fitted times
    assert ttft > 0 and executed > 0
    assert off <= 0.02  # int8 of normal values: half a step of max/127 is 1.5% of their norm at most


def test_every_batch_is_the_schedulers(ex):
    # the engine's batches by the step rule: budget and seats are kept, a prompt's chunks come before its decode
    e = ex.Engine(budget=64, seqs=4, layers=1, blocks=64, block=8, q_heads=4, kv_heads=2, dim=64, fmt="16")
    for prompt, out in ((100, 3), (5, 2), (70, 1), (1, 4), (40, 2)):
        e.submit(prompt, out)
    total = [100 + 5 + 70 + 1 + 40, 3 + 2 + 1 + 4 + 2]
    while e.waiting or e.running:
        n = len(e.log)
        e.step()
        F = e.log[n][0]
        assert F[0] == 1 and 0 < F[1] + F[2] <= 64 and F[2] <= 4
    assert [sum(f[i] for f, _ in e.log) for i in (1, 2)] == total
    assert len(e.free) == 64 and e.cache.status() == 0
