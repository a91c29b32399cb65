"""examples/engine_batches.py and the router: the estimates are of the batches that the engine executes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_engine_example import ex  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompt", [1, 511, 512, 1300])
def test_an_estimate_counts_the_batches_that_are_executed(ex, prompt):
    # the router's features of a new prompt on the engine's state are those of the batches up to its first token, one by one
    # added up: whole numbers, so equal
    e = ex.Engine(budget=512, seqs=6, layers=1, blocks=900, block=8, q_heads=4, kv_heads=2, dim=64, fmt="e4m3")
    for p, out in ((900, 30), (5, 20), (600, 11), (1, 40), (333, 2)):
        e.submit(p, out)
    for _ in range(4):
        e.step()
    assert e.running
    coef = np.array([[1e-3, 1e-6, 2e-6, 1e-8, 3e-9]], np.float32)
    rt = ex.router_of(e, coef)
    rt.load_state(*ex.snapshot(e))
    p = torch.tensor([prompt], dtype=torch.int32, device="cuda")
    want = rt.estimate_features(p)[0, 0].tolist()
    ttft = float(rt.estimate_ttft(p)[0, 0])
    assert rt.status() == 0
    rt.close()
    n = len(e.log)
    e.submit(prompt, 4)
    mine = e.waiting[-1]
    while mine[2] == 4:
        e.step()
    got = np.sum([f for f, _ in e.log[n:]], axis=0).tolist()
    assert got == want
    # Eq. 9 is linear in them: fp32 products and sums of five positive terms
    assert abs(ttft - float(np.dot(coef[0].astype(np.float64), want))) <= 16 * 2.0 ** -24 * ttft


def test_the_fit_recovers_what_the_log_was_made_of(ex):
    # times that are Eq. 9 of the logged features exactly: the coefficients come back
    e = ex.Engine(budget=512, seqs=6, layers=1, blocks=900, block=8, q_heads=4, kv_heads=2, dim=64, fmt="e4m3")
    for i in range(14):
        e.submit(1 + 377 * i % 1050, 3 + 11 * i % 40)
    while e.waiting or e.running:
        e.step()
    coef = np.array([1e-3, 2e-6, 5e-6, 3e-8, 1e-8])
    e.log = [(f, float(np.dot(coef, f))) for f, _ in e.log]
    got = ex.fit(e)[0]
    F = np.array([f for f, _ in e.log], np.float64)
    assert np.abs(F @ got - F @ coef).max() <= 1e-6 * (F @ coef).max()
