"""One instance's token batches, executed, timed and fitted: from the engine's kernels to the router's estimates.

The simulation behind the router counts token batches and costs each by Eq. 9, whose coefficients are
fitted to a log of executed batches (Sec. 4.1).  This example makes such a log.  A small engine serves prompts
FCFS under a token budget and a sequence cap with chunked prefill -- the scheduler's step rule --, keeps
their K and V in a paged cache (lr_cache_write) and attends over it (lr_cache_attend), a number of layers a batch.
The time of every batch and its features go to lr_calibrate; a router created with the fitted
coefficients then estimates the time to first token of one more prompt on the engine's state, and
the engine serves it.  Last, a sequence is handed to a second cache of another format: read back as values
(lr_cache_read) and stored there.

    python examples/engine_batches.py [--layers 16] [--format e4m3]

The tensors are random: no model is involved, and only the attention's part of a layer is executed.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_18253_gb300 import cache as C  # noqa: E402
from paper_2607_18253_gb300 import router as R  # noqa: E402

FORMATS = {"16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def make_cache(blocks, block, kv_heads, dim, q_heads, fmt, max_seqs):
    shape = (blocks, block, kv_heads, dim)
    kv = [torch.zeros(shape, dtype=FORMATS[fmt], device="cuda") for _ in range(2)]
    sc = [None if fmt == "16" else torch.ones(shape[:3], device="cuda") for _ in range(2)]
    return C.PagedCache(k=kv[0], v=kv[1], k_scale=sc[0], v_scale=sc[1], num_q_heads=q_heads, dtype=torch.bfloat16, max_seqs=max_seqs)


class Engine:
    """An instance: running requests [context, prompt tokens left, output tokens left, blocks], a waiting queue, a cache."""

    def __init__(self, *, budget, seqs, layers, blocks, block=16, q_heads=32, kv_heads=8, dim=128, fmt="e4m3", seed=0):
        self.budget, self.seqs, self.layers, self.block = budget, seqs, layers, block
        self.q_heads, self.kv_heads, self.dim = q_heads, kv_heads, dim
        self.cache = make_cache(blocks, block, kv_heads, dim, q_heads, fmt, seqs)
        self.free = list(range(blocks - 1, -1, -1))
        self.running, self.waiting, self.log = [], [], []
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        # a fused projection's output for the largest batch: queries, keys, values
        self.qkv = torch.randn((budget, q_heads + 2 * kv_heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        self.out = torch.empty((budget, q_heads, dim), dtype=torch.bfloat16, device="cuda")
        self.table = np.zeros((seqs, blocks), np.int32)
        self.clock = 0.0

    def submit(self, prompt, output):
        self.waiting.append([0, prompt, output, []])

    def schedule(self):
        """The next batch: (request, tokens) in running order, then waiting requests while budget and seats last."""
        left, batch = self.budget, []
        for r in self.running:
            n = min(r[1], left) if r[1] > 0 else min(1, left)
            if n > 0:
                batch.append((r, n))
                left -= n
        while left > 0 and self.waiting and len(self.running) < self.seqs:
            r = self.waiting.pop(0)
            self.running.append(r)
            n = min(r[1], left)
            batch.append((r, n))
            left -= n
        return batch

    def step(self):
        """Executes one batch."""
        batch = self.schedule()
        if not batch:
            return
        q, kv, F = [], [], [1, 0, 0, 0, 0]
        for i, (r, n) in enumerate(batch):
            while len(r[3]) * self.block < r[0] + n:
                r[3].append(self.free.pop())
            self.table[i, :len(r[3])] = r[3]
            q.append(n)
            kv.append(r[0] + n)
            if r[1] > 0:
                F[1] += n
                F[4] += n * r[0] + n * (n + 1) // 2
            else:
                F[2] += 1
                F[3] += r[0]
        T, width = sum(q), max(len(r[3]) for r, _ in batch)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
        b = C.CacheBatch(dev(np.concatenate([[0], np.cumsum(q)])), dev(kv), dev(self.table[:len(q), :width]), max(q))
        x = self.qkv[:T]
        qs, ks, vs = x[:, :self.q_heads], x[:, self.q_heads:self.q_heads + self.kv_heads], x[:, self.q_heads + self.kv_heads:]
        graph = torch.cuda.CUDAGraph()  # as engines do: the batch's launches cost the host nothing
        with torch.cuda.graph(graph):
            for _ in range(self.layers):  # (one cache stands for every layer's)
                self.cache.write(ks, vs, b)
                self.cache.attend(qs, b, out=self.out[:T])
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        graph.replay()
        t1.record()
        t1.synchronize()
        seconds = t0.elapsed_time(t1) * 1e-3
        self.clock += seconds
        self.log.append((F, seconds))
        for r, n in batch:
            r[0] += n
            if r[1] > 0:
                r[1] -= n
            else:
                r[2] -= 1
        for r in [r for r in self.running if r[1] == 0 and r[2] <= 0]:
            self.running.remove(r)
            self.free.extend(r[3])


def fit(engine):
    """Eq. 9 coefficients of the engine's log, through a one-instance router context."""
    F = torch.tensor([f for f, _ in engine.log], dtype=torch.int64, device="cuda")
    t = torch.tensor([s for _, s in engine.log], dtype=torch.float64, device="cuda")
    rt = router_of(engine, np.zeros((1, 5), np.float32))
    coef = rt.calibrate(F, torch.zeros(len(t), dtype=torch.int32, device="cuda"), t, shared_beta1=False).cpu().numpy()
    if rt.status() != R.LR_OK:
        raise RuntimeError("calibration")
    rt.close()
    return coef


def router_of(engine, coef):
    return R.LatencyRouter(model_of_instance=[0], coef=np.maximum(coef, 0).astype(np.float32), price_in=[0.0], price_out=[0.0],
                           max_batched_tokens=[engine.budget], max_seqs=[engine.seqs], cap_running=engine.seqs, cap_waiting=64,
                           max_queries=16, max_prompt_len=8192)


def snapshot(engine):
    """The engine's requests as lr_load_state takes them."""
    R_, W = engine.seqs, 64
    n_run, n_wait = np.array([len(engine.running)]), np.array([len(engine.waiting)])
    run, wait = np.zeros((3, 1, R_)), np.ones((2, 1, W))
    run[2] = 1
    for i, r in enumerate(engine.running):
        run[0, 0, i], run[1, 0, i], run[2, 0, i] = r[0], r[1], max(1, r[2])
    for i, r in enumerate(engine.waiting):
        wait[0, 0, i], wait[1, 0, i] = r[1], max(1, r[2])
    arrays = (n_run, run[0], run[1], run[2], n_wait, wait[0], wait[1])
    return [torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda() for a in arrays]


def hand_over(engine, fmt):
    """The first running request's cached tokens in a new cache of format `fmt`: (values here, values there)."""
    r = engine.running[0]
    n = r[0]
    i32 = dict(dtype=torch.int32, device="cuda")
    span, length = torch.tensor([0, n], **i32), torch.tensor([n], **i32)
    here = C.CacheBatch(span, length, torch.tensor([r[3]], **i32), n)
    k, v = engine.cache.read(here, n)
    blocks = -(-n // engine.block)
    other = make_cache(blocks, engine.block, engine.kv_heads, engine.dim, engine.q_heads, fmt, 1)
    there = C.CacheBatch(span, length, torch.arange(blocks, **i32)[None], n)
    other.write(k, v, there)
    got = other.read(there, n)
    if engine.cache.status() != R.LR_OK or other.status() != R.LR_OK:
        raise RuntimeError("hand-over")
    other.close()
    return (k, v), got


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=16)
    ap.add_argument("--budget", type=int, default=2048)
    ap.add_argument("--seqs", type=int, default=64)
    ap.add_argument("--prompts", type=int, default=120)
    ap.add_argument("--format", choices=list(FORMATS), default="e4m3")
    a = ap.parse_args(argv)
    rng = np.random.default_rng(0)
    e = Engine(budget=a.budget, seqs=a.seqs, layers=a.layers, blocks=a.seqs * 640, fmt=a.format)
    for _ in range(a.prompts):
        e.submit(int(np.clip(rng.lognormal(np.log(512), 1.0), 1, 4096)), int(rng.integers(8, 120)))
    e.step()
    e.log.clear()  # (the first batch pays for the first launches)
    while e.waiting or len(e.running) > a.seqs // 2:
        e.step()
    if e.cache.status() != R.LR_OK:
        raise RuntimeError("engine")
    coef = fit(e)
    F = np.array([f for f, _ in e.log], np.float64)
    t = np.array([s for _, s in e.log])
    mape = float(np.mean(np.abs(F @ coef[0] - t) / t))
    print(f"{len(t)} batches, {1e3 * t.mean():.3f} ms on average; fitted coefficients "
          f"{', '.join('%.3g' % c for c in coef[0])} s; mean error of the fit {100 * mape:.1f}%")
    prompt = 1500
    rt = router_of(e, coef)
    rt.load_state(*snapshot(e))
    ttft = float(rt.estimate_ttft(torch.tensor([prompt], dtype=torch.int32, device="cuda"))[0, 0])
    if rt.status() != R.LR_OK:
        raise RuntimeError("estimate")
    rt.close()
    before = e.clock
    e.submit(prompt, 4)
    mine = e.waiting[-1]
    while mine[2] == 4:
        e.step()
    print(f"time to first token of a prompt of {prompt}: estimated {1e3 * ttft:.3f} ms, executed {1e3 * (e.clock - before):.3f} ms")
    (k, v), (k2, v2) = hand_over(e, "int8")
    off = float((k2.float() - k.float()).norm() / k.float().norm())
    print(f"a sequence of {k.shape[0]} tokens handed over, {a.format} to int8: values within {100 * off:.2f}%")
    return coef, mape, ttft, e.clock - before, off


if __name__ == "__main__":
    main()
