"""Paged KV cache and its attention on the GPU against plain implementations in 64 bits.

Stored codes and scales are elementwise fp32 formulas, so they are compared exactly.  An attention
output is sum_j w_j v_j with w = softmax: against 64 bits it may differ by
  u |o|             its own rounding (u = 2^-8 bf16, 2^-11 fp16)
  u A               the weights' rounding for the second product, A = sum_j w_j |v_j|
  e A               fp32 arithmetic: a score is off by at most 2^-24 (D + 8) S (S = scale sum_d |q_d k_d|, at its
                    largest), a weight by twice that and the exponential's 2^-21, the sums by 2^-24 a term
  n 2^-25 V         fp16 weights below its normal range (V = max |v|, n terms), and the output's 2^-25
The bound below is the sum of these; lse is off by the scores' error and 2^-20.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def C():
    from paper_2607_18253_gb300 import cache
    return cache


def R():
    from paper_2607_18253_gb300 import router
    return router


def quantised(x, fmt):
    """(codes, scale) of fp32 vectors [..., D] by the formulas of the header."""
    top = torch.tensor(448.0 if fmt == "e4m3" else 127.0, device=x.device)
    a = x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100)
    y = x * (top.expand_as(a).contiguous() / a)
    if fmt == "e4m3":
        c = y.clamp(-448, 448).to(torch.float8_e4m3fn)
    else:
        c = y.round().clamp(-127, 127).nan_to_num(0.0).to(torch.int8)
    return c, (a / top.expand_as(a).contiguous()).squeeze(-1)


class Case:
    """A cache with random contents, a batch of sequences (q_len, kv_len) and its handle."""

    def __init__(self, seqs, *, H=2, G=4, D=128, b=16, dtype="bf16", fmt="16", heads_first=False, seed=0, spare=5,
                 q_std=1.5, pad=0, garbage=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.seqs, self.H, self.G, self.D, self.b, self.dt, self.fmt = seqs, H, G, D, b, dtype, fmt
        n = len(seqs)
        nblk = [-(-kv // b) for _, kv in seqs]
        self.nb = sum(nblk) + spare
        order = torch.randperm(self.nb, device="cuda", generator=g, dtype=torch.int64)
        width = max([1] + nblk)
        self.table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for s in range(n):
            self.table[s, :nblk[s]] = order[at:at + nblk[s]].to(torch.int32)
            at += nblk[s]
        shape = (self.nb, H, b, D) if heads_first else (self.nb, b, H, D)
        turn = (lambda t: t.transpose(1, 2)) if heads_first else (lambda t: t)
        self.k_scale = self.v_scale = None
        x = [torch.randn(shape, device="cuda", generator=g).to(DT[dtype]) for _ in range(2)]
        if fmt == "16":
            self.k, self.v = (turn(t) for t in x)
        else:
            q = [quantised(t.float(), fmt) for t in x]
            (self.k, self.k_scale), (self.v, self.v_scale) = ((turn(c), turn(s)) for c, s in q)
        self.T = sum(q for q, _ in seqs)
        self.q = (torch.randn((self.T + pad, H * G, D), device="cuda", generator=g) * q_std).to(DT[dtype])
        self.q_start = torch.tensor([0] + list(np.cumsum([q for q, _ in seqs])), dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor([kv for _, kv in seqs], dtype=torch.int32, device="cuda")
        if garbage is not None:  # every place that is no token's
            used = torch.zeros(self.nb, b, dtype=torch.bool, device="cuda")
            for s in range(n):
                p = torch.arange(seqs[s][1], device="cuda")
                used[self.table[s].long()[p // b], p % b] = True
            for t, sc in ((self.k, self.k_scale), (self.v, self.v_scale)):
                (t if sc is None else sc)[~used] = garbage
        self.batch = C().CacheBatch(self.q_start, self.kv_len, self.table, max([1] + [q for q, _ in seqs]))
        self.cache = C().PagedCache(k=self.k, v=self.v, k_scale=self.k_scale, v_scale=self.v_scale, num_q_heads=H * G,
                                    dtype=DT[dtype], max_seqs=max(1, n))

    def values(self, which, s, h, n):
        """fp64 values of the first n tokens of sequence s, head h."""
        p = torch.arange(n, device="cuda")
        blk, off = self.table[s].long()[p // self.b], p % self.b
        t, sc = (self.k, self.k_scale) if which == "k" else (self.v, self.v_scale)
        if sc is None:
            return t[blk, off, h].double()
        return t.view(torch.int8)[blk, off, h].view(t.dtype).double() * sc[blk, off, h].double()[:, None]

    def reference(self, scale=None, window=0, sinks=0):
        """(out, lse, bound of out, bound of lse) in fp64."""
        scale = self.D ** -0.5 if scale is None else scale
        H, G, D, u = self.H, self.G, self.D, U[self.dt]
        out = torch.zeros(self.T, H * G, D, dtype=torch.float64, device="cuda")
        lse = torch.full((self.T, H * G), -math.inf, dtype=torch.float64, device="cuda")
        tol, ltol = torch.full_like(out, 1e-30), torch.zeros_like(lse)
        t0 = 0
        for s, (ql, kv) in enumerate(self.seqs):
            rows = slice(t0, t0 + ql)
            t0 += ql
            if kv == 0 or ql == 0:
                continue
            at = torch.arange(kv - ql, kv, device="cuda")[:, None]
            j = torch.arange(kv, device="cuda")[None, :]
            see = j <= at
            if window:
                see &= (j > at - window) | (j < sinks)
            for h in range(H):
                k, v = self.values("k", s, h, kv), self.values("v", s, h, kv)
                q = self.q[rows, h * G:(h + 1) * G].double()
                x = torch.einsum("tgd,jd->tgj", q, torch.nan_to_num(k, 0.0, 0.0, 0.0)) * scale
                big = float((torch.einsum("tgd,jd->tgj", q.abs(), torch.nan_to_num(k.abs(), 0.0, 0.0, 0.0)) * scale).amax())
                x = x.masked_fill(~see[:, None, :], -math.inf)
                l = torch.logsumexp(x, -1)
                w = torch.where(see[:, None, :], torch.exp(x - l[..., None]), torch.zeros_like(x)).nan_to_num(0.0)
                # (what a row does not see is left out, whatever it is)
                v0 = torch.nan_to_num(v, 0.0, 0.0, 0.0)
                o, A = w @ v0, w @ v0.abs()
                sc = 2.0 ** -24 * (D + 8) * big
                e = 2 * sc + 2.0 ** -21 + 2.0 ** -24 * (kv + 64)
                out[rows, h * G:(h + 1) * G], lse[rows, h * G:(h + 1) * G] = o, l
                small = (kv + 1) * 2.0 ** -25 * (float(v0.abs().max()) + 1.0) if self.dt == "fp16" else 0.0
                tol[rows, h * G:(h + 1) * G] = u * o.abs() + (u + e) * A * 1.01 + small + 1e-30
                ltol[rows, h * G:(h + 1) * G] = sc + 2.0 ** -20 * (1 + l.abs().nan_to_num(0.0, 0.0, 0.0))
        return out, lse, tol, ltol

    def check(self, window=0, sinks=0, scale=None, **kw):
        out, lse = self.cache.attend(self.q, self.batch, scale=scale, window=window, sinks=sinks, lse=True, **kw)
        torch.cuda.synchronize()
        assert self.cache.status() == R().LR_OK
        ref, rl, tol, ltol = self.reference(scale, window, sinks)
        out, lse = out[:self.T].double(), lse[:self.T].double()
        assert torch.isfinite(out).all()
        over = (out - ref).abs() / tol
        assert float(over.max() if over.numel() else 0.0) <= 1.0, float(over.max())
        empty = torch.isinf(rl)
        assert torch.equal(empty, torch.isinf(lse) & (lse < 0))
        assert not out[empty].any()
        d = (lse - rl).abs()[~empty]
        assert not d.numel() or bool((d <= ltol[~empty]).all())
        return out, lse


# ---------------------------------------------------------------------------------------------
# store and load

@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D,b,heads_first", [(1, 16, 1, False), (3, 80, 7, True), (8, 128, 16, False), (5, 64, 33, True)])
def test_store_and_load_are_exact(fmt, dtype, H, D, b, heads_first):
    seqs = [(1, 1), (5, 17), (0, 9), (40, 40), (1, 130), (33, 77)]
    c = Case(seqs, H=H, G=2, D=D, b=b, dtype=dtype, fmt=fmt, heads_first=heads_first, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn((c.T, 3 * H, D), device="cuda", generator=g)
    x[::3] *= 1e-3
    x[1::5] *= 300.0
    x[2] = 0.0
    x = x.to(DT[dtype])
    k, v = x[:, H:2 * H], x[:, 2 * H:]  # slices of a fused projection
    before = [t.clone() if t is not None else None for t in (c.k, c.v, c.k_scale, c.v_scale)]
    c.cache.write(k, v, c.batch)
    got = c.cache.read(c.batch, c.T)
    got32 = c.cache.read(c.batch, c.T, torch.float32)
    assert c.cache.status() == R().LR_OK
    blk, off = [], []
    for s, (ql, kv) in enumerate(seqs):
        p = torch.arange(kv - ql, kv, device="cuda")
        blk.append(c.table[s].long()[p // b])
        off.append(p % b)
    blk, off = torch.cat(blk), torch.cat(off)
    for new, t, sc, t0, s0, val, val32 in ((k, c.k, c.k_scale, before[0], before[2], got[0], got32[0]),
                                           (v, c.v, c.v_scale, before[1], before[3], got[1], got32[1])):
        raw = torch.int16 if fmt == "16" else torch.int8
        if fmt == "16":
            want, want32 = new, new.float()
        else:
            want, ws = quantised(new.float(), fmt)
            want32 = want.float() * ws[..., None]
            assert torch.equal(sc[blk, off], ws)
            s0[blk, off] = ws
            assert torch.equal(sc, s0)
        assert torch.equal(t.view(raw)[blk, off], want.contiguous().view(raw))
        t0.view(raw)[blk, off] = want.contiguous().view(raw)
        assert torch.equal(t.view(raw), t0.view(raw))  # nothing else is touched
        assert torch.equal(val32, want32)
        assert torch.equal(val, want32.to(DT[dtype]))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_vectors_that_are_not_finite_read_back_as_nan(fmt):
    c = Case([(6, 20)], H=2, G=1, D=64, fmt=fmt, seed=5)
    k = torch.randn((6, 2, 64), device="cuda").to(torch.bfloat16)
    v = k.clone()
    k[1, 0, 7], k[2, 1, 9], v[3, 0, 0] = math.inf, math.nan, -math.inf
    c.cache.write(k, v, c.batch)
    rk, rv = c.cache.read(c.batch, 6)
    assert c.cache.status() == R().LR_OK
    bad_k, bad_v = torch.zeros(6, 2, dtype=torch.bool), torch.zeros(6, 2, dtype=torch.bool)
    bad_k[1, 0] = bad_k[2, 1] = bad_v[3, 0] = True
    for got, bad in ((rk, bad_k), (rv, bad_v)):
        assert torch.equal(torch.isnan(got).all(-1).cpu(), bad) and torch.equal(torch.isnan(got).any(-1).cpu(), bad)


def test_rows_without_a_place():
    # more new tokens than kv_len, a block out of range, a position past the table: recorded, nothing stored;
    # rows of no sequence are left as they are
    c = Case([(4, 20), (3, 18), (2, 12)], H=1, G=1, D=32, b=8, seed=6, pad=5)
    c.table[1, 2] = c.nb  # position 17 (the third block)
    kv = c.kv_len.clone()
    kv[2] = 1
    batch = C().CacheBatch(c.q_start, kv, c.table, 8)
    k0, v0 = c.k.clone(), c.v.clone()
    x = torch.randn((c.T + 5, 1, 32), device="cuda").to(torch.bfloat16)
    c.cache.write(x, x, batch)
    assert c.cache.status() == R().LR_EINVAL
    out = tuple(torch.full((c.T + 5, 1, 32), 9.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    c.cache.read(batch, c.T + 5, out=out)
    assert c.cache.status() == R().LR_EINVAL
    assert c.cache.status() == R().LR_OK  # cleared
    lost = [4 + 1, 4 + 2, 7]  # positions 16, 17 of the second sequence and -1 of the third
    keep = [i for i in range(c.T) if i not in lost]
    for o in out:
        assert torch.isnan(o[lost]).all() and torch.equal(o[keep], x[keep]) and bool((o[c.T:] == 9.0).all())
    changed = ((c.k != k0) | (c.v != v0)).any(-1).sum()
    assert int(changed) <= len(keep)


# ---------------------------------------------------------------------------------------------
# attention

SEQS = {
    "one": [(1, 1)],
    "singles": [(1, 1), (1, 63), (1, 64), (1, 65), (1, 500), (1, 17)],
    "chunks": [(5, 5), (64, 300), (33, 64), (2, 129)],
    "mixed": [(1, 77), (0, 10), (130, 200), (1, 1), (3, 1000)],
    "empty": [(4, 2), (3, 0), (1, 0), (70, 66)],
}


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", list(SEQS))
def test_attention(fmt, dtype, seqs):
    Case(SEQS[seqs], dtype=dtype, fmt=fmt, seed=11).check()


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("G,D,b,heads_first", [(1, 64, 1, False), (3, 80, 5, True), (8, 16, 16, False), (16, 96, 24, False),
                                               (17, 128, 64, True), (40, 64, 128, False)])
def test_head_layouts(fmt, G, D, b, heads_first):
    for seqs in (SEQS["singles"], SEQS["mixed"]):
        Case(seqs, H=3, G=G, D=D, b=b, fmt=fmt, heads_first=heads_first, seed=12).check()


@pytest.mark.parametrize("fmt", ["16", "int8"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (64, 200), (100, 64), (129, 1), (4000, 3),
                                          (1 << 30, 1 << 30)])
def test_window_and_sinks(fmt, window, sinks):
    for seqs in (SEQS["singles"], SEQS["mixed"], [(200, 700), (1, 699)], SEQS["empty"]):
        Case(seqs, D=64, fmt=fmt, seed=13).check(window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_sharp_and_flat_softmax(dtype):
    Case(SEQS["mixed"], dtype=dtype, seed=14, q_std=30.0).check()
    Case(SEQS["mixed"], dtype=dtype, seed=15).check(scale=1e-6)
    Case(SEQS["mixed"], dtype=dtype, seed=16).check(scale=2.0)


@pytest.mark.parametrize("fmt", ["16", "e4m3"])
@pytest.mark.parametrize("seqs", [[(1, 40001)], [(1, 20000), (1, 3), (2, 9000)], [(300, 5000)], [(1, 30 + 7 * i) for i in range(300)]])
def test_tokens_split_over_the_gpu(fmt, seqs):
    c = Case(seqs, H=2, G=4, fmt=fmt, seed=17)
    a, la = c.check()
    b, lb = c.check()
    assert torch.equal(a, b) and torch.equal(la, lb)  # joined in one order


@pytest.mark.parametrize("fmt", ["16", "int8"])
def test_more_sequences_than_threads(fmt):
    # 1,500 sequences, some without new tokens, one chunk among them: every round of the walks over a batch
    seqs = [(1 if i % 7 else 0, 1 + i % 90) for i in range(1499)]
    seqs.insert(700, (70, 200))
    c = Case(seqs, H=1, G=2, D=64, fmt=fmt, seed=27)
    c.check()
    x = torch.randn((c.T, 1, 64), device="cuda").to(torch.bfloat16)
    c.cache.write(x, x, c.batch)
    k, v = c.cache.read(c.batch, c.T)
    assert c.cache.status() == R().LR_OK and torch.equal(k, v)
    want = x
    if fmt != "16":
        codes, sc = quantised(x.float(), fmt)
        want = (codes.float() * sc[..., None]).to(torch.bfloat16)
    assert torch.equal(k, want)


def test_strided_queries_and_outputs():
    c = Case(SEQS["mixed"], H=2, G=4, D=64, seed=18)
    T = c.T
    wide = torch.zeros((T, 3, 8, 64), device="cuda", dtype=torch.bfloat16)
    wide[:, 1] = c.q
    out = torch.full((T, 8, 2, 64), 5.0, device="cuda", dtype=torch.bfloat16)
    want, _ = c.cache.attend(c.q, c.batch)
    c.cache.attend(wide[:, 1], c.batch, out=out[:, :, 1])
    assert torch.equal(out[:, :, 1], want) and bool((out[:, :, 0] == 5.0).all())
    turned = torch.empty((8, T, 64), device="cuda", dtype=torch.bfloat16).copy_(c.q.transpose(0, 1)).transpose(0, 1)
    got, _ = c.cache.attend(turned, c.batch)
    assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_places_that_are_no_tokens_do_not_matter(fmt, value):
    for seqs in (SEQS["singles"], SEQS["mixed"], SEQS["empty"]):
        Case(seqs, fmt=fmt, seed=19, garbage=value).check()


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("ql,kv,window,sinks,where", [(40, 100, 0, 0, 80), (200, 300, 0, 0, 250), (1, 300, 50, 4, 240),
                                                      (90, 300, 50, 4, 170), (300, 300, 20, 2, 100)])
def test_tokens_that_a_row_does_not_see_do_not_reach_it(fmt, value, ql, kv, window, sinks, where):
    # K and V of one position are not finite: the rows that see it get NaN or infinities, the others what they would
    c = Case([(ql, kv), (3, 50)], H=2, G=4, D=64, fmt=fmt, seed=20)
    ref, _, tol, _ = c.reference(window=window, sinks=sinks)
    blk, off = int(c.table[0, where // c.b]), where % c.b
    for which in ("v", "k"):
        t, sc = (c.k, c.k_scale) if which == "k" else (c.v, c.v_scale)
        x = t if fmt == "16" else sc
        keep = x[blk, off].clone()
        x[blk, off] = value
        out = c.cache.attend(c.q, c.batch, window=window, sinks=sinks)[0].double()
        assert c.cache.status() == R().LR_OK
        at = torch.arange(kv - ql, kv, device="cuda")
        sees = at >= where
        if window:
            sees &= (where > at - window) | (where < sinks)
        sees = torch.cat([sees, torch.zeros(3, dtype=torch.bool, device="cuda")])
        assert bool((~torch.isfinite(out[sees])).all()) if which == "v" else bool((~torch.isfinite(out[sees])).any() or not sees.any())
        assert torch.isfinite(out[~sees]).all()
        assert bool(((out - ref).abs() <= tol)[~sees].all())
        x[blk, off] = keep


def test_hidden_blocks_are_not_looked_up():
    # an engine frees the blocks that a window has passed: their table entries may be anything
    c = Case([(1, 1000), (5, 700)], D=64, seed=21)
    want = c.cache.attend(c.q, c.batch, window=100, sinks=4)[0]
    c.table[0, 1:56] = -7
    c.table[1, 1:37] = 1 << 30
    got = c.cache.attend(c.q, c.batch, window=100, sinks=4)[0]
    assert c.cache.status() == R().LR_OK and torch.equal(got, want)


def test_blocks_out_of_range_are_reported():
    for seqs in ([(1, 300), (1, 200)], [(90, 300), (1, 200)]):
        c = Case(seqs, D=64, seed=22)
        want = c.cache.attend(c.q, c.batch)[0]
        c.table[0, 3] = c.nb
        got = c.cache.attend(c.q, c.batch)[0]
        assert c.cache.status() == R().LR_EINVAL
        n = seqs[0][0]
        assert torch.isnan(got[:n]).all() and torch.equal(got[n:], want[n:])


def test_sequences_out_of_range_are_left_out():
    c = Case([(2, 50), (3, 60), (1, 40)], D=64, seed=23, pad=4)
    want = c.cache.attend(c.q, c.batch)[0]
    for q_start, kv, max_q in (([0, 2, 5, 6], [50, -1, 40], 3), ([0, 2, 5, 6], [50, 10 ** 6, 40], 3),
                               ([0, 2, 5, 6], [50, 60, 40], 2)):
        out = torch.full_like(c.q, 7.0)
        b = C().CacheBatch(torch.tensor(q_start, dtype=torch.int32, device="cuda"),
                           torch.tensor(kv, dtype=torch.int32, device="cuda"), c.table, max_q)
        c.cache.attend(c.q, b, out=out)
        assert c.cache.status() == R().LR_EINVAL
        assert torch.equal(out[:2], want[:2]) and torch.equal(out[5:6], want[5:6])
        assert bool((out[2:5] == 7.0).all()) and bool((out[6:] == 7.0).all())


def test_offsets_past_32_bits():
    # a cache of more than 2^32 bytes a tensor: the sequence lives in its last blocks, which a wrapped offset misses
    H, D, b = 8, 128, 64
    nb = (5 << 30) // (H * D * b * 2)
    k = torch.zeros((nb, b, H, D), device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    kv, last = 300, torch.arange(nb - 5, nb, device="cuda", dtype=torch.int32)[None]
    cache = C().PagedCache(k=k, v=v, num_q_heads=16, max_seqs=1)
    new_k, new_v = (torch.randn((kv, H, D), device="cuda").to(torch.bfloat16) for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda")
    whole = C().CacheBatch(torch.tensor([0, kv], **i32), torch.tensor([kv], **i32), last, kv)
    cache.write(new_k, new_v, whole)
    rk, rv = cache.read(whole, kv)
    assert torch.equal(rk, new_k) and torch.equal(rv, new_v)
    assert torch.equal(k[nb - 5:].reshape(-1, H, D)[:kv], new_k)
    assert not k[:nb - 5].any()
    q = torch.randn((200, 16, D), device="cuda").to(torch.bfloat16)
    for n in (1, 200):
        out, _ = cache.attend(q[:n], C().CacheBatch(torch.tensor([0, n], **i32), torch.tensor([kv], **i32), last, n))
        x = torch.einsum("thgd,jhd->thgj", q[:n].view(n, H, 2, D).double(), new_k.double()) * D ** -0.5
        at = torch.arange(kv - n, kv, device="cuda")
        x = x.masked_fill(torch.arange(kv, device="cuda")[None, None, None] > at[:, None, None, None], -math.inf)
        ref = torch.einsum("thgj,jhd->thgd", x.softmax(-1), new_v.double()).reshape(n, 16, D)
        assert float((out.double() - ref).abs().max()) < 0.05  # (a wrong block gives zeros or another's values: off by 0.3 and more)
    assert cache.status() == R().LR_OK
    cache.close()


def test_another_stream_and_a_graph():
    c = Case(SEQS["mixed"], D=64, seed=24)
    want = c.cache.attend(c.q, c.batch)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros_like(c.q)
    c.cache.attend(c.q, c.batch, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    x = torch.randn((c.T, c.H, 64), device="cuda").to(torch.bfloat16)
    c.cache.write(x, x, c.batch)
    want = c.cache.attend(c.q, c.batch)[0]
    torch.cuda.synchronize()
    graph, got = torch.cuda.CUDAGraph(), torch.zeros_like(c.q)
    with torch.cuda.graph(graph):
        c.cache.write(x, x, c.batch)
        c.cache.attend(c.q, c.batch, out=got)
    got.zero_()
    c.k.zero_()
    # (the whole cache was cleared: only the batch's own tokens come back)
    graph.replay()
    torch.cuda.synchronize()
    again = c.cache.attend(c.q, c.batch)[0]
    assert torch.equal(got, again) and not torch.equal(got, want)


def test_nothing_to_do():
    c = Case([(1, 10)], D=64, seed=25)
    i32 = dict(dtype=torch.int32, device="cuda")
    none = C().CacheBatch(torch.zeros(1, **i32), torch.zeros(0, **i32), torch.zeros((0, 1), **i32), 1)
    q = c.q[:0]
    assert c.cache.attend(q, none)[0].shape == (0, 8, 64)
    assert c.cache.read(none, 0)[0].shape == (0, 2, 64)
    out = torch.full_like(c.q, 3.0)
    c.cache.attend(c.q, none, out=out)  # rows, but of no sequence
    idle = C().CacheBatch(torch.zeros(2, **i32), c.kv_len, c.table, 1)
    c.cache.attend(c.q, idle, out=out)
    assert bool((out == 3.0).all()) and c.cache.status() == R().LR_OK


# ---------------------------------------------------------------------------------------------
# refusals

def test_refused_configurations():
    k = torch.zeros((4, 16, 2, 64), device="cuda", dtype=torch.bfloat16)
    make = lambda **kw: C().PagedCache(**{**dict(k=k, v=k.clone(), num_q_heads=8), **kw})  # noqa: E731
    make().close()
    codes = torch.zeros((4, 16, 2, 64), device="cuda", dtype=torch.int8)
    sc = torch.zeros((4, 16, 2), device="cuda")
    for kw in (dict(num_q_heads=7), dict(num_q_heads=0), dict(num_q_heads=2050), dict(max_seqs=0), dict(max_seqs=1 << 20),
               dict(k=k[..., :24], v=k[..., :24]), dict(k=k[..., 4:36], v=k[..., 4:36]),
               dict(k=torch.zeros((4, 16, 2, 144), device="cuda", dtype=torch.bfloat16),
                    v=torch.zeros((4, 16, 2, 144), device="cuda", dtype=torch.bfloat16)),
               dict(k=torch.zeros((1, 5000, 2, 16), device="cuda", dtype=torch.bfloat16),
                    v=torch.zeros((1, 5000, 2, 16), device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(R().LRError) as e:
            make(**kw)
        assert e.value.code == R().LR_EINVAL
    for kw in (dict(dtype=torch.float32), dict(k=k.float(), v=k.float()), dict(k=k.cpu(), v=k.cpu()), dict(v=codes), dict(v=k[:2]),
               dict(k=codes, v=codes), dict(k=codes, v=codes, k_scale=sc.double(), v_scale=sc.double()),
               dict(k=codes, v=codes, k_scale=sc[:2], v_scale=sc[:2]), dict(k=k[0], v=k[0])):
        with pytest.raises((TypeError, ValueError)):
            make(**kw)


def test_refused_calls():
    c = Case([(2, 30), (1, 20)], H=2, G=4, D=64, seed=26)
    q, b = c.q, c.batch
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(sinks=-1),
               dict(window=(1 << 30) + 1)):
        with pytest.raises(R().LRError) as e:
            c.cache.attend(q, b, **kw)
        assert e.value.code == R().LR_EINVAL
    for bad in (q.float(), q[:, :4], q.cpu(), q[..., :32], q.transpose(1, 2)):
        with pytest.raises((TypeError, ValueError)):
            c.cache.attend(bad, b)
    with pytest.raises((TypeError, ValueError)):
        c.cache.attend(q, b, out=q[:1])
    with pytest.raises((TypeError, ValueError)):
        c.cache.write(q[:, :2], q[:, :3], b)
    with pytest.raises(R().LRError):
        c.cache.read(b, 3, dtype=torch.float16)
    odd = torch.zeros((3, 8, 68), device="cuda", dtype=torch.bfloat16)
    for bad in (odd[..., :64], odd[..., 1:65]):  # strides and starts that are no multiple of 16 bytes
        with pytest.raises(R().LRError) as e:
            c.cache.attend(bad, b)
        assert e.value.code == R().LR_EINVAL
    i32 = dict(dtype=torch.int32, device="cuda")
    many = C().CacheBatch(torch.zeros(4, **i32), torch.zeros(3, **i32), torch.zeros((3, 2), **i32), 1)
    for call in (lambda: c.cache.attend(q, many), lambda: c.cache.write(q[:, :2], q[:, :2], many), lambda: c.cache.read(many, 1)):
        with pytest.raises(R().LRError) as e:
            call()
        assert e.value.code == R().LR_ECAPACITY
    with pytest.raises(R().LRError):
        c.cache.attend(q, C().CacheBatch(c.q_start, c.kv_len, c.table, 0))
    with pytest.raises(R().LRError):
        c.cache.attend(q, C().CacheBatch(c.q_start, c.kv_len, c.table, (1 << 20) + 1))
    with pytest.raises((TypeError, ValueError)):
        C().CacheBatch(c.q_start.long(), c.kv_len, c.table, 2)
    with pytest.raises((TypeError, ValueError)):
        C().CacheBatch(c.q_start, c.kv_len, c.table.t(), 2)
    assert c.cache.status() == R().LR_OK
    lib = R().load_library()
    assert lib.lr_cache_destroy(None) == R().LR_OK
    assert lib.lr_cache_attend(None, None, 1, None, 0, 0, 1.0, 0, 0, None, 0, 0, None, None) == R().LR_EINVAL
    assert lib.lr_cache_last_error(None) == b""
