"""Trees of drafted tokens over the paged cache, and which tokens it keeps, on the GPU against plain implementations in 64 bits.

Attention of a tree is bounded as in test_gpu_cache.py: the same sums, over the tokens that a row's mask names.

A weight is w = decay w0 + sum_r p_r with p_r = exp(x_r - lse_r), lse as the call is given it.  In fp32
  a score is off by 2^-24 (D + 8) S (S = scale sum_d |q_d k_d|, at its largest), over 8 bits by 2^-24 max|q| scale sum_d |k_d|
    more (bf16 queries in fp16), and by 2^-23 (|x| + |lse|) for its factors and its difference from lse, in units of log2
  p_r is off by that much of itself and the exponential's 2^-21
  the sums by 2^-24 a term
and the bound is p's share summed, with the terms' rounding.  Choices and moves are compared exactly.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_cache as base  # noqa: E402
from test_gpu_cache import C, DT, R, SEQS, _built  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------
# trees

class Tree(base.Case):
    """masks: "tree" (ancestors of random parents), "any" (random bits, in any order), "none"."""

    def __init__(self, seqs, masks="tree", words=None, tree_seed=0, **kw):
        super().__init__(seqs, **kw)
        rng = np.random.default_rng(tree_seed)
        most = max([1] + [q for q, _ in seqs])
        self.words = -(-most // 32) if words is None else words
        self.paths = []
        rows = []
        for q, _ in seqs:
            see = np.zeros((q, self.words * 32), bool)
            for i in range(q):
                if masks == "tree":
                    if i and rng.random() < 0.95:
                        see[i] = see[rng.integers(0, i)]
                    see[i, i] = True
                elif masks == "any":
                    see[i, :q] = rng.random(q) < rng.choice([0.05, 0.5, 0.95])
            self.paths.append(torch.from_numpy(see[:, :q].copy()).cuda())
            see[:, q:] = rng.random((q, self.words * 32 - q)) < 0.5  # bits of no token
            rows.append(np.packbits(see, axis=1, bitorder="little").view(np.int32))
        pad = np.full((self.q.shape[0] - self.T, self.words), -1, np.int32)
        self.tree = torch.from_numpy(np.concatenate(rows + [pad])).cuda()

    def sees(self, s, window, sinks):
        """[rows, tokens] of sequence s."""
        ql, kv = self.seqs[s]
        see = torch.cat([torch.ones((ql, kv - ql), dtype=torch.bool, device="cuda"), self.paths[s]], 1)
        if window:
            place = see.long().cumsum(1) - 1
            see &= (place > place[:, -1:] - window) | (place < sinks)
        return see

    def reference(self, scale=None, window=0, sinks=0):
        scale = self.D ** -0.5 if scale is None else scale
        H, G, D, u = self.H, self.G, self.D, base.U[self.dt]
        out = torch.zeros(self.T, H * G, D, dtype=torch.float64, device="cuda")
        lse = torch.full((self.T, H * G), -math.inf, dtype=torch.float64, device="cuda")
        tol, ltol = torch.full_like(out, 1e-30), torch.zeros_like(lse)
        t0 = 0
        for s, (ql, kv) in enumerate(self.seqs):
            rows = slice(t0, t0 + ql)
            t0 += ql
            if ql == 0:
                continue
            see = self.sees(s, window, sinks)[:, None, :]
            for h in range(H):
                heads = slice(h * G, (h + 1) * G)
                k, v = self.values("k", s, h, kv), self.values("v", s, h, kv)
                q = self.q[rows, heads].double()
                k0, v0 = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
                x = torch.einsum("tgd,jd->tgj", q, k0) * scale
                big = float((torch.einsum("tgd,jd->tgj", q.abs(), k0.abs()) * scale).amax())
                x = x.masked_fill(~see, -math.inf)
                l = torch.logsumexp(x, -1)
                w = torch.where(see, torch.exp(x - l[..., None]), torch.zeros_like(x)).nan_to_num(0.0)
                o, A = w @ v0, w @ v0.abs()
                sc = 2.0 ** -24 * (D + 8) * big
                e = 2 * sc + 2.0 ** -21 + 2.0 ** -24 * (kv + 64)
                out[rows, heads], lse[rows, heads] = o, l
                small = (kv + 1) * 2.0 ** -25 * (float(v0.abs().max()) + 1.0) if self.dt == "fp16" else 0.0
                tol[rows, heads] = u * o.abs() + (u + e) * A * 1.01 + small + 1e-30
                ltol[rows, heads] = sc + 2.0 ** -20 * (1 + l.abs().nan_to_num(0.0, 0.0, 0.0))
        return out, lse, tol, ltol

    def check(self, window=0, sinks=0, scale=None, **kw):
        return super().check(window, sinks, scale, tree=self.tree, **kw)


TREES = {
    "one": [(1, 1)],
    "few": [(1, 1), (2, 65), (2, 2), (1, 500), (2, 129)],           # the kernel of few rows
    "small": [(4, 40), (16, 16), (9, 700), (1, 33), (13, 128)],
    "wide": [(64, 64), (200, 1000), (33, 161), (1, 90), (0, 12), (129, 300)],
}


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", list(TREES))
def test_trees(fmt, dtype, seqs):
    Tree(TREES[seqs], dtype=dtype, fmt=fmt, seed=41).check()


@pytest.mark.parametrize("masks", ["any", "none"])
@pytest.mark.parametrize("seqs", list(TREES))
def test_masks_of_any_kind(masks, seqs):
    # tokens before and behind a row's own, itself left out; rows that see the context alone, or nothing
    Tree(TREES[seqs], masks=masks, seed=42).check()
    Tree([(q, q) for q, _ in TREES[seqs]], masks=masks, seed=43, G=2, D=64, fmt="int8").check()


@pytest.mark.parametrize("fmt", ["16", "e4m3"])
@pytest.mark.parametrize("G,D,b,heads_first", [(1, 64, 1, False), (3, 80, 5, True), (8, 16, 16, False), (16, 96, 24, False),
                                               (17, 128, 64, True), (6, 128, 8, True)])
def test_tree_head_layouts(fmt, G, D, b, heads_first):
    for seqs in ("few", "wide"):
        Tree(TREES[seqs], H=3, G=G, D=D, b=b, fmt=fmt, heads_first=heads_first, seed=44).check()


@pytest.mark.parametrize("masks", ["tree", "any"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (3, 2), (16, 4), (16, 40), (100, 64), (129, 1), (4000, 3), (1 << 30, 1 << 30)])
def test_tree_window_and_sinks(masks, window, sinks):
    for seqs, G in (("few", 2), ("small", 1), ("wide", 4)):
        Tree(TREES[seqs], masks=masks, G=G, D=64, seed=45, tree_seed=window).check(window=window, sinks=sinks)
    Tree([(16, 30), (16, 16), (5, 600)], masks=masks, H=2, G=1, fmt="int8", seed=46).check(window=window, sinks=sinks)


def test_a_chain_is_causal():
    # each token's ancestors are all before it: the causal call's own result
    for seqs, fmt in ((TREES["small"], "16"), ([(70, 900)], "e4m3"), (TREES["few"], "int8")):
        c = Tree(seqs, fmt=fmt, seed=47)
        rows = [np.packbits(np.tril(np.ones((q, c.words * 32), bool)), axis=1, bitorder="little").view(np.int32) for q, _ in seqs]
        chain = torch.from_numpy(np.concatenate(rows)).cuda()
        for window, sinks in ((0, 0), (37, 3)):
            want, wl = c.cache.attend(c.q, c.batch, window=window, sinks=sinks, lse=True)
            got, gl = c.cache.attend(c.q, c.batch, window=window, sinks=sinks, lse=True, tree=chain)
            assert torch.allclose(gl, wl, rtol=2.0 ** -18, atol=2.0 ** -18)
            u = base.U["bf16"]
            assert bool(((got.double() - want.double()).abs() <= 3 * u * c.v.float().abs().max() * 5 + 1e-30).all()) if fmt == "16" else True


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_hidden_tokens_do_not_reach_a_row(fmt, value):
    # a drafted token that no other row sees, and every place that is no token's
    for seqs in ([(8, 700), (3, 40), (2, 2)], [(2, 300), (1, 5)]):
        c = Tree(seqs, seed=48, garbage=value, fmt=fmt)
        t0 = 0
        for s, (q, kv) in enumerate(seqs):
            last = c.paths[s][:, q - 1].clone()
            c.paths[s][:, q - 1] = False
            for r in range(q):
                c.tree[t0 + r, (q - 1) // 32] &= ~(1 << (q - 1) % 32)
            blk, at = int(c.table[s, (kv - 1) // c.b]), (kv - 1) % c.b
            for t, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
                (t if sc is None else sc)[blk, at] = value
            t0 += q
            assert last.any()
        c.check()


@pytest.mark.parametrize("fmt", ["16", "e4m3"])
@pytest.mark.parametrize("seqs", [[(40, 60001)], [(9, 20000), (1, 3), (33, 9000)], [(8, 30000)], [(100, 40000), (70, 40000)],
                                  [(30, 12000)], [(17, 5000), (32, 3001), (1, 64)]])
def test_trees_split_over_the_gpu(fmt, seqs):
    # few and many parts of a unit, joined at once or by groups: the same bits every time
    c = Tree(seqs, H=1, G=4, fmt=fmt, seed=73)
    a, la = c.check()
    b, lb = c.check()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_tree_rows_and_strides():
    # more words than needed, rows of a wider tensor, rows of no sequence, one mask for all rows
    c = Tree(TREES["wide"], words=9, seed=49, pad=7)
    wide = torch.full((c.T + 7, 20), -1, dtype=torch.int32, device="cuda")
    wide[:, 3:12] = c.tree
    want, wl = c.cache.attend(c.q, c.batch, tree=c.tree, lse=True)
    out = torch.full_like(c.q, 7.0)
    lse = torch.full((c.T + 7, c.q.shape[1]), 7.0, device="cuda")
    c.cache.attend(c.q, c.batch, tree=wide[:, 3:12], out=out, lse=lse)
    assert c.cache.status() == R().LR_OK
    assert torch.equal(out[:c.T], want[:c.T]) and torch.equal(lse[:c.T], wl[:c.T])
    assert bool((out[c.T:] == 7.0).all()) and bool((lse[c.T:] == 7.0).all())
    one = c.tree[:1].expand(c.T + 7, 9)
    a, _ = c.cache.attend(c.q, c.batch, tree=one)
    b, _ = c.cache.attend(c.q, c.batch, tree=one.contiguous())
    assert torch.equal(a[:c.T], b[:c.T])


def test_tree_errors():
    c = Tree([(4, 40), (8, 80), (3, 3)], seed=50)
    want, _ = c.cache.attend(c.q, c.batch, tree=c.tree)
    kv = c.kv_len.clone()
    kv[2] = 2  # fewer tokens than it brings
    table = c.table.clone()
    table[1, 0] = c.nb  # rows of the second sequence read it
    out = torch.full_like(c.q, 3.0)
    c.cache.attend(c.q, C().CacheBatch(c.q_start, kv, table, 8), tree=c.tree, out=out)
    assert c.cache.status() == R().LR_EINVAL and c.cache.status() == R().LR_OK
    assert torch.equal(out[:4], want[:4]) and torch.isnan(out[4:12]).all() and bool((out[12:] == 3.0).all())
    with pytest.raises(R().LRError, match="tree_words"):
        c.cache.attend(c.q, C().CacheBatch(c.q_start, c.kv_len, c.table, 33), tree=c.tree)
    with pytest.raises(TypeError, match="tree"):
        c.cache.attend(c.q, c.batch, tree=c.tree.long())
    with pytest.raises(ValueError, match="tree"):
        c.cache.attend(c.q, c.batch, tree=c.tree[:-1])


# ---------------------------------------------------------------------------------------------
# weights

def weights_of(c, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.rand(c.k.shape[:3], device="cuda", generator=g)


def expected(c, lse, w0, decay, window=0, sinks=0, scale=None):
    """(weights, bound) in fp64 over the whole cache."""
    scale = c.D ** -0.5 if scale is None else scale
    w, tol = w0.double().clone(), torch.zeros_like(w0, dtype=torch.float64)
    t0 = 0
    for s, (ql, kv) in enumerate(c.seqs):
        rows = slice(t0, t0 + ql)
        t0 += ql
        if ql == 0 or kv == 0:
            continue
        at = torch.arange(kv - ql, kv, device="cuda")[:, None]
        j = torch.arange(kv, device="cuda")
        see = j <= at
        if window:
            see &= (j > at - window) | (j < sinks)
        blk, place = c.table[s].long()[j // c.b], j % c.b
        for h in range(c.H):
            k, q = c.values("k", s, h, kv), c.q[rows, h * c.G:(h + 1) * c.G].double()
            l = lse[rows, h * c.G:(h + 1) * c.G].double()
            x = torch.einsum("tgd,jd->tgj", q, k) * scale
            off = 2.0 ** -24 * (c.D + 8) * float((torch.einsum("tgd,jd->tgj", q.abs(), k.abs()) * scale).amax())
            if c.fmt != "16" and c.dt == "bf16":
                off += 2.0 ** -24 * scale * float(q.abs().max()) * float(k.abs().sum(-1).max())
            off = off + 2.0 ** -23 * (x.abs() + l.abs()[..., None].nan_to_num(0.0, 0.0, 0.0))
            hit = see[:, None] & (l > -math.inf)[..., None]
            p = torch.where(hit, torch.exp(x - torch.where(l > -math.inf, l, 0.0)[..., None]), torch.zeros_like(x))
            new = p.sum((0, 1)) + (decay * w[blk, place, h] * (j < kv - ql) if decay else 0.0)
            tol[blk, place, h] = (p * (1.01 * off + 2.0 ** -21)).sum((0, 1)) + 2.0 ** -24 * (ql * c.G + 8) * new.abs() + 2.0 ** -126
            w[blk, place, h] = new
    return w, tol


def check_weights(c, decay=1.0, window=0, sinks=0, w0=None, scale=None):
    w0 = weights_of(c) if w0 is None else w0
    _, lse = c.cache.attend(c.q, c.batch, lse=True, window=window, sinks=sinks, scale=scale)
    w = w0.clone()
    assert c.cache.weigh(c.q, lse, c.batch, w, decay=decay, window=window, sinks=sinks, scale=scale) is w
    assert c.cache.status() == R().LR_OK
    want, tol = expected(c, lse, w0, decay, window, sinks, scale)
    over = (w.double() - want).abs() > tol
    assert not over.any(), (int(over.sum()), float((w.double() - want).abs().max()))
    return w


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", list(SEQS))
def test_weigh(fmt, dtype, seqs):
    c = base.Case(SEQS[seqs], dtype=dtype, fmt=fmt, seed=51)
    for decay in (1.0, 0.0, 0.9375):
        check_weights(c, decay)


@pytest.mark.parametrize("fmt", ["16", "e4m3"])
@pytest.mark.parametrize("G,D,b,heads_first", [(1, 64, 1, False), (3, 80, 5, True), (8, 16, 16, False), (16, 96, 24, False),
                                               (17, 128, 64, True), (40, 64, 128, False)])
def test_weigh_head_layouts(fmt, G, D, b, heads_first):
    for seqs in (SEQS["singles"], SEQS["mixed"]):
        check_weights(base.Case(seqs, H=3, G=G, D=D, b=b, fmt=fmt, heads_first=heads_first, seed=52), 0.5)


@pytest.mark.parametrize("decay", [1.0, 0.25])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 200), (129, 1), (300, 17), (1 << 30, 1 << 30)])
def test_weigh_window_and_sinks(decay, window, sinks):
    for seqs in (SEQS["singles"], SEQS["mixed"], [(200, 700), (1, 699)], [(700, 900)], SEQS["empty"]):
        for fmt in ("16", "int8"):
            check_weights(base.Case(seqs, D=64, fmt=fmt, seed=53), decay, window, sinks)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("seqs", [[(1, 40001)], [(300, 5000)], [(2500, 2500)], [(1, 30 + 7 * i) for i in range(300)], [(40, 9000), (1, 3), (130, 2000)]])
def test_weigh_is_the_same_every_time(fmt, seqs):
    c = base.Case(seqs, H=2, G=4, fmt=fmt, seed=54)
    w0 = weights_of(c)
    assert torch.equal(check_weights(c, w0=w0), check_weights(c, w0=w0))


def test_weigh_many_rows_of_one_head():
    check_weights(base.Case([(1500, 1700)], H=1, G=8, seed=55))
    check_weights(base.Case([(700, 700), (900, 5000)], H=1, G=1, D=80, fmt="e4m3", dtype="fp16", seed=56), 0.0)


@pytest.mark.parametrize("fmt", ["16", "int8"])
def test_more_sequences_than_threads(fmt):
    # every round of the walks over a batch, in either kernel, and of the lists
    seqs = [(1 if i % 7 else 0, 1 + i % 90) for i in range(1299)]
    seqs.insert(900, (70, 200))
    c = base.Case(seqs, H=1, G=2, D=64, fmt=fmt, seed=74)
    w = check_weights(c, 0.5)
    kept, count = choose(c, w, 40, sinks=1, recent=7)
    check_keep(c, kept, count, w=w)
    Tree([(1 + i % 3, 5 + i % 60) for i in range(1200)] + [(50, 90)], H=1, G=2, D=64, fmt=fmt, seed=75).check()


def test_weigh_sharp_rows_and_scale():
    c = base.Case(SEQS["mixed"], seed=57, q_std=20.0)
    check_weights(c)
    check_weights(c, scale=0.7)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("seqs", [SEQS["singles"], SEQS["mixed"], [(140, 500)]])
def test_weigh_leaves_other_places_alone(fmt, seqs):
    # places that are no token's hold NaN in the cache and in the weights; new tokens' and, with decay 0, all old weights are not read
    for value in (math.nan, math.inf):
        c = base.Case(seqs, fmt=fmt, seed=58, garbage=value, H=3)
        w0 = torch.full(c.k.shape[:3], math.nan, device="cuda")
        used = torch.zeros(c.nb, c.b, dtype=torch.bool, device="cuda")
        old = used.clone()
        for s, (ql, kv) in enumerate(seqs):
            p = torch.arange(kv if ql else 0, device="cuda")
            used[c.table[s].long()[p // c.b], p % c.b] = True
            p = p[:max(0, kv - ql)]
            old[c.table[s].long()[p // c.b], p % c.b] = True
        _, lse = c.cache.attend(c.q, c.batch, lse=True)
        w = w0.clone()
        c.cache.weigh(c.q, lse, c.batch, w, decay=0.0)
        assert torch.isfinite(w[used]).all() and torch.isnan(w[~used]).all()
        w0[old] = 0.5
        w = w0.clone()
        c.cache.weigh(c.q, lse, c.batch, w)
        assert torch.isfinite(w[used]).all() and torch.isnan(w[~used]).all()
        assert c.cache.status() == R().LR_OK


def test_weigh_layouts_of_weights_and_queries():
    c = base.Case(SEQS["mixed"], H=3, G=4, D=64, seed=59)
    _, lse = c.cache.attend(c.q, c.batch, lse=True)
    w0 = weights_of(c)
    want = c.cache.weigh(c.q, lse, c.batch, w0.clone())
    turned = w0.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(c.cache.weigh(c.q, lse, c.batch, turned), want)
    wide = torch.zeros((*w0.shape, 3), device="cuda")
    wide[..., 1] = w0
    qs = torch.zeros((c.T, 3, 12, 64), device="cuda", dtype=torch.bfloat16)
    qs[:, 2] = c.q
    assert torch.equal(c.cache.weigh(qs[:, 2], lse, c.batch, wide[..., 1]), want)
    assert not wide[..., ::2].any()


def test_weigh_errors():
    c = base.Case([(2, 40), (8, 80), (3, 30)], seed=60)
    _, lse = c.cache.attend(c.q, c.batch, lse=True)
    w0 = weights_of(c)
    want = c.cache.weigh(c.q, lse, c.batch, w0.clone())
    kv, table = c.kv_len.clone(), c.table.clone()
    kv[0] = 1 << 29   # more than its blocks hold: left out
    table[1, 1] = -5  # tokens 16 .. 31 of the second have no place
    w = c.cache.weigh(c.q, lse, C().CacheBatch(c.q_start, kv, table, 8), w0.clone())
    assert c.cache.status() == R().LR_EINVAL and c.cache.status() == R().LR_OK
    want[c.table[0].long()[:3]] = w0[c.table[0].long()[:3]]
    want[c.table[1, 1].long()] = w0[c.table[1, 1].long()]
    assert torch.equal(w, want)
    with pytest.raises(R().LRError, match="decay"):
        c.cache.weigh(c.q, lse, c.batch, w, decay=-1.0)
    with pytest.raises(R().LRError, match="decay"):
        c.cache.weigh(c.q, lse, c.batch, w, decay=math.nan)
    with pytest.raises(TypeError, match="weights"):
        c.cache.weigh(c.q, lse, c.batch, w.double())
    with pytest.raises(ValueError, match="weights"):
        c.cache.weigh(c.q, lse, c.batch, w[1:])
    with pytest.raises(ValueError):
        c.cache.weigh(c.q, lse[1:], c.batch, w)


def test_rows_that_saw_nothing_add_nothing():
    c = base.Case([(1, 70), (20, 50)], seed=61)
    _, lse = c.cache.attend(c.q, c.batch, lse=True)
    w0 = weights_of(c)
    lse[0], lse[5:] = -math.inf, -math.inf
    w = c.cache.weigh(c.q, lse, c.batch, w0.clone())
    want, tol = expected(c, lse, w0, 1.0)
    assert bool(((w.double() - want).abs() <= tol).all())


# ---------------------------------------------------------------------------------------------
# choice and move

def chosen(w, m, sinks, recent):
    """Positions kept of a list of weights (numpy)."""
    kv = len(w)
    p = np.arange(kv)
    must = (p < sinks) | (p >= kv - recent)
    rank = np.where(np.isnan(w), np.inf, w)
    order = np.lexsort((p, -rank, ~np.isnan(w), ~must))
    order = np.concatenate([p[must], order[must.sum():]])
    return np.sort(order[:m])


def choose(c, w, cap, budget=None, sinks=0, recent=0):
    kept, count = c.cache.select(w, c.batch, cap, budget=budget, sinks=sinks, recent=recent)
    assert c.cache.status() == R().LR_OK
    assert kept.shape == (len(c.seqs), c.H, cap) and kept.dtype == torch.int32
    host, hw, table = kept.cpu().numpy(), w.cpu().numpy(), c.table.cpu().numpy()
    for s, (_, kv) in enumerate(c.seqs):
        m = min(kv, cap if budget is None else int(budget[s]))
        assert int(count[s]) == m
        p = np.arange(kv)
        for h in range(c.H):
            want = chosen(hw[table[s][p // c.b], p % c.b, h], m, sinks, recent)
            assert np.array_equal(host[s, h, :m], want), (s, h)
            assert (host[s, h, m:] == -1).all()
    return kept, count


LISTS = [(1, 1), (1, 31), (1, 32), (1, 33), (1, 0), (1, 700), (1, 511), (1, 513), (1, 5000)]


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("cap,sinks,recent", [(1, 0, 0), (64, 4, 16), (512, 0, 0), (600, 16, 255), (513, 513, 0), (100, 0, 100), (6000, 4, 64)])
def test_select(cap, sinks, recent, heads_first):
    c = base.Case(LISTS, H=3, G=1, D=16, b=24 if heads_first else 16, heads_first=heads_first, seed=62)
    w = torch.exp(3.0 * torch.randn(c.k.shape[:3], device="cuda") - 4.0)
    if heads_first:
        w = w.transpose(1, 2).contiguous().transpose(1, 2)
    choose(c, w, cap, sinks=sinks, recent=recent)
    budget = torch.tensor([min(cap, (37 * i + sinks + recent) % (cap + 1)) for i in range(len(LISTS))], dtype=torch.int32, device="cuda")
    choose(c, w, cap, budget=budget, sinks=sinks, recent=recent)


@pytest.mark.parametrize("kind", ["equal", "few", "near", "signs", "special"])
def test_select_ties_and_values(kind):
    c = base.Case([(1, 3000), (1, 100), (1, 4097)], H=2, G=1, D=16, seed=63)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    n = torch.randn(c.k.shape[:3], device="cuda", generator=g)
    w = {"equal": torch.full_like(n, 0.25), "few": torch.floor(n * 2.0), "near": 1.0 + (n * 3).round() * 2.0 ** -23,
         "signs": torch.where(n.abs() < 0.5, torch.copysign(torch.zeros_like(n), n), n), "special": n}[kind]
    if kind == "special":
        for i, v in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -math.nan)):
            w[torch.rand(n.shape, device="cuda", generator=g) < 0.05] = v
    for cap in (1, 50, 99, 777, 2999):
        choose(c, w, cap, sinks=min(cap, 3))


def test_select_of_long_lists():
    # more than a CTA's keys, more than a cluster's
    c = base.Case([(1, 250001), (1, 120000)], H=1, G=1, D=16, b=64, seed=64)
    w = torch.rand(c.k.shape[:3], device="cuda")
    choose(c, w, 20000, sinks=4, recent=1024)
    choose(c, torch.floor(w * 8), 130000)
    choose(c, torch.full_like(w, 1.0), 33333, recent=1)
    # a CTA an SM, sixteen a list
    c = base.Case([(1, 900001)], H=1, G=1, D=16, b=128, seed=77)
    w = torch.rand(c.k.shape[:3], device="cuda")
    choose(c, w, 300000, sinks=1)
    check_keep(c, *lists(c, 300000, share=0.3), w=w)


def moved(c, kept, count, start, w):
    """What keep gives, by a host loop over whole lists."""
    got = {"k": c.k.clone(), "v": c.v.clone(), "ks": c.k_scale, "vs": c.v_scale, "w": w}
    got = {n: t.clone() for n, t in got.items() if t is not None}
    for s in range(len(c.seqs)):
        m, at = int(count[s]), int(start[s]) if start is not None else 0
        for h in range(c.H):
            src = (kept[s, h] if kept.dim() == 3 else kept[s])[:m].long()
            dst = torch.arange(at, at + m, device="cuda")
            t = c.table[s].long()
            for x in got.values():
                x = x.view(torch.int8) if x.dtype == torch.float8_e4m3fn else x
                x[t[dst // c.b], dst % c.b, h] = x[t[src // c.b], src % c.b, h]
    return got


def check_keep(c, kept, count, start=None, w=None):
    want = moved(c, kept, count, start, w)
    c.cache.keep(kept, count, c.batch, weights=w, start=start)
    assert c.cache.status() == R().LR_OK
    for n, t in {"k": c.k, "v": c.v, "ks": c.k_scale, "vs": c.v_scale, "w": w}.items():
        if t is not None:
            raw = {1: torch.int8, 2: torch.int16, 4: torch.int32}[t.element_size()]
            assert torch.equal(t.contiguous().view(raw), want[n].contiguous().view(raw)), n


def lists(c, cap, seed=0, heads=True, start=None, share=None):
    """Random ascending lists."""
    rng = np.random.default_rng(seed)
    n, H = len(c.seqs), c.H
    kept, count = np.full((n, H, cap), -1, np.int32), np.zeros(n, np.int32)
    for s, (_, kv) in enumerate(c.seqs):
        at = 0 if start is None else int(start[s])
        most = min(cap, kv - at)
        count[s] = rng.integers(0, most + 1) if share is None else min(most, round(share * kv))
        for h in range(H):
            kept[s, h, :count[s]] = np.sort(at + rng.permutation(kv - at)[:count[s]])
    if not heads:
        kept = kept[:, 0]
    return torch.from_numpy(np.ascontiguousarray(kept)).cuda(), torch.from_numpy(count).cuda()


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("H,D,b,heads_first", [(1, 16, 1, False), (3, 80, 7, True), (8, 128, 16, False), (5, 64, 33, True), (2, 96, 64, False)])
def test_keep(fmt, H, D, b, heads_first):
    for cap, heads, seqs in ((9, True, LISTS), (700, True, LISTS), (5000, False, LISTS), (64, False, [(1, 2)])):
        c = base.Case(seqs, H=H, G=1, D=D, b=b, fmt=fmt, heads_first=heads_first, seed=65)
        check_keep(c, *lists(c, cap, heads=heads), w=weights_of(c))
        start = torch.tensor([kv // 3 for _, kv in seqs], dtype=torch.int32, device="cuda")
        check_keep(c, *lists(c, cap, seed=1, heads=heads, start=start), start=start)


@pytest.mark.parametrize("fmt", ["16", "int8"])
@pytest.mark.parametrize("share", [0.02, 0.3, 0.7, 0.97, 1.0])
def test_keep_long_lists_in_place(fmt, share):
    # every chunk of a list is written where others are read
    seqs = [(1, 60001), (1, 4000), (1, 7)]
    c = base.Case(seqs, H=2, G=1, D=128, fmt=fmt, seed=66)
    for _ in range(3):
        check_keep(c, *lists(c, 60001, share=share, seed=int(share * 100)), w=weights_of(c))
    # the same distance for all tokens: the last of a chunk is next to the first of another
    kept = torch.arange(1, 4000, device="cuda", dtype=torch.int32)
    kept = torch.stack([kept, kept, kept])
    check_keep(c, kept, torch.tensor([3999, 3999, 6], dtype=torch.int32, device="cuda"))


def test_keep_errors():
    # lists that do not ascend, lie below their place or behind the tokens; counts and starts out of range; no block
    c = base.Case([(1, 50), (1, 40), (1, 30), (1, 20), (1, 60)], H=2, G=1, D=32, seed=67)
    kept = torch.full((5, 2, 4), -1, dtype=torch.int32, device="cuda")
    kept[0, 0] = torch.tensor([3, 2, 50, 49])   # place 1 not ascending, place 2 behind the tokens, place 3 not above its neighbour
    kept[0, 1] = torch.tensor([0, 1, 2, 9])
    kept[1:] = torch.tensor([5, 6, 7, 8])
    kept[4, :, 2:] = torch.tensor([17, 33])
    count = torch.tensor([4, 5, 2, 2, 4], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 0, -1, 19, 0], dtype=torch.int32, device="cuda")
    table = c.table.clone()
    table[4, 1] = c.nb + 3
    k0 = c.k.clone()
    c.cache.keep(kept, count, C().CacheBatch(c.q_start, c.kv_len, table, 1), start=start)
    assert c.cache.status() == R().LR_EINVAL and c.cache.status() == R().LR_OK
    want = k0.clone()
    want[c.table[0, 0], 0, 0] = k0[c.table[0, 0], 3, 0]
    want[c.table[0, 0], 3, 1] = k0[c.table[0, 0], 9, 1]
    for i, p in ((0, 5), (1, 6)):
        want[c.table[4, 0], i] = k0[c.table[4, 0], p]
    want[c.table[4, 0], 3] = k0[c.table[4, 2], 1]
    assert torch.equal(c.k, want)
    with pytest.raises(ValueError, match="kept"):
        c.cache.keep(kept[:, :1], count, c.batch)
    with pytest.raises(ValueError):
        c.cache.keep(kept, count[1:], c.batch)
    with pytest.raises(TypeError):
        c.cache.keep(kept.long(), count, c.batch)


def test_select_errors():
    c = base.Case([(1, 50), (1, 40), (1, 30)], H=2, G=1, D=32, seed=68)
    w = weights_of(c) + 1.0
    kv, table = c.kv_len.clone(), c.table.clone()
    kv[0] = 1 << 30
    table[1, 0] = -1  # its 16 tokens have the lowest weight
    budget = torch.tensor([5, 24, 9], dtype=torch.int32, device="cuda")
    batch = C().CacheBatch(c.q_start, kv, table, 1)
    kept, count = c.cache.select(w, batch, 24, budget=budget)
    assert c.cache.status() == R().LR_EINVAL and c.cache.status() == R().LR_OK
    assert count.tolist() == [0, 24, 9] and bool((kept[0] == -1).all())
    assert bool((kept[1] == torch.arange(16, 40, device="cuda")).all())
    budget[2] = 25
    _, count = c.cache.select(w, c.batch, 24, budget=budget)
    assert c.cache.status() == R().LR_EINVAL and count.tolist() == [5, 24, 0]
    for kw in (dict(sinks=20, recent=5), dict(sinks=-1), dict(recent=-1)):
        with pytest.raises(R().LRError):
            c.cache.select(w, c.batch, 24, **kw)
    with pytest.raises(R().LRError):
        c.cache.select(w, c.batch, -1)


# ---------------------------------------------------------------------------------------------
# together

@pytest.mark.parametrize("fmt,dtype", [("16", "bf16"), ("e4m3", "bf16"), ("int8", "fp16")])
def test_prompts_are_cut_down_and_decoded(fmt, dtype):
    # prompts store their tokens, the last rows weigh them, each head keeps what it used most, decoding goes on over what is left
    c = base.Case([(300, 300), (32, 900), (40, 40)], H=2, G=4, dtype=dtype, fmt=fmt, seed=69)
    g = torch.Generator(device="cuda")
    g.manual_seed(70)
    c.cache.write(*(torch.randn((c.T, 2, 128), device="cuda", generator=g).to(DT[dtype]) for _ in range(2)), c.batch)
    w = torch.zeros(c.k.shape[:3], device="cuda")
    w = check_weights(c, 0.0, w0=w)
    kept, count = choose(c, w, 128, sinks=4, recent=16)
    check_keep(c, kept, count, w=w)
    kv = [int(n) + 1 for n in count]
    d = base.Case.__new__(base.Case)
    d.__dict__.update(c.__dict__)
    d.seqs, d.T, d.q = [(1, n) for n in kv], 3, c.q[:3].contiguous()
    d.q_start = torch.arange(4, dtype=torch.int32, device="cuda")
    d.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
    d.batch = C().CacheBatch(d.q_start, d.kv_len, d.table, 1)
    d.cache.write(*(torch.randn((3, 2, 128), device="cuda", generator=g).to(DT[dtype]) for _ in range(2)), d.batch)
    d.check()
    check_weights(d, 1.0, w0=w)


def test_a_tree_is_verified_and_its_path_kept():
    c = Tree([(8, 100), (5, 37), (16, 16)], H=2, G=2, seed=71)
    out, _ = c.check()
    paths, starts = [], []
    for s, (q, kv) in enumerate(c.seqs):
        deep = int(c.paths[s].sum(1).argmax())
        paths.append((kv - q) + torch.nonzero(c.paths[s][deep]).flatten())
        starts.append(kv - q)
    kept = torch.full((3, 16), -1, dtype=torch.int32, device="cuda")
    for s, p in enumerate(paths):
        kept[s, :len(p)] = p.to(torch.int32)
    count = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    check_keep(c, kept, count, start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    # the deepest row's attention, now of an ordinary last token
    last = torch.stack([c.q[int(c.q_start[s]) + int(c.paths[s].sum(1).argmax())] for s in range(3)])
    kv_len = torch.tensor([a + len(p) for a, p in zip(starts, paths)], dtype=torch.int32, device="cuda")
    batch = C().CacheBatch(torch.arange(4, dtype=torch.int32, device="cuda"), kv_len, c.table, 1)
    got, _ = c.cache.attend(last, batch)
    want = torch.stack([out[int(c.q_start[s]) + int(c.paths[s].sum(1).argmax())] for s in range(3)])
    # two roundings of the output and two of the weights, of values whose weighted magnitudes are at most max |v|
    assert bool(((got.double() - want).abs() <= 4.1 * base.U["bf16"] * float(c.v.abs().max())).all())


def test_offsets_beyond_32_bits():
    # 4.6 GB of K and of V, the sequences' blocks anywhere in them
    c = Tree([(8, 300), (3, 90), (40, 700)], H=8, G=2, spare=140000, seed=78)
    assert c.k.numel() * 2 > 1 << 32 and int(c.table.max()) * c.k.stride(0) * 2 > 1 << 32
    c.check()
    w = check_weights(c, 0.5)
    check_weights(Tree([(1, 300), (2, 90)], H=8, G=2, spare=140000, seed=79))
    kept, count = choose(c, w, 128, sinks=2, recent=8)
    check_keep(c, kept, count, w=w)


def test_calls_on_two_streams():
    # each with a cache of its own, at the same time: lists that clusters move, joined parts
    cases = [Tree([(40, 30000), (3, 700)], H=2, G=4, fmt=fmt, seed=76) for fmt in ("16", "e4m3")]
    streams = [torch.cuda.Stream() for _ in cases]
    plan = [lists(c, 30000, share=0.4, seed=3) for c in cases]
    want, got = [], []
    for c, (kept, count) in zip(cases, plan):
        state = [t.clone() for t in (c.k, c.v)]
        w = weights_of(c)
        out, lse = c.cache.attend(c.q, c.batch, lse=True, tree=c.tree)
        c.cache.weigh(c.q, lse, c.batch, w)
        c.cache.keep(kept, count, c.batch, weights=w)
        want.append([out, lse, w, c.k.clone(), c.v.clone()])
        c.k.copy_(state[0])
        c.v.copy_(state[1])
        if c.k_scale is not None:
            want[-1] += [c.k_scale.clone()]
    scales = [None if c.k_scale is None else base.Case([(40, 30000), (3, 700)], H=2, G=4, fmt=c.fmt, seed=76) for c in cases]
    for c, fresh in zip(cases, scales):
        if fresh is not None:
            c.k_scale.copy_(fresh.k_scale)
            c.v_scale.copy_(fresh.v_scale)
    torch.cuda.synchronize()
    for c, st, (kept, count) in zip(cases, streams, plan):
        with torch.cuda.stream(st):
            w = weights_of(c)
            out, lse = c.cache.attend(c.q, c.batch, lse=True, tree=c.tree)
            c.cache.weigh(c.q, lse, c.batch, w)
            c.cache.keep(kept, count, c.batch, weights=w, stream=st)
            got.append([out, lse, w, c.k, c.v] + ([c.k_scale] if c.k_scale is not None else []))
    torch.cuda.synchronize()
    for c, x, y in zip(cases, want, got):
        assert c.cache.status() == R().LR_OK
        for t, u in zip(x, y):
            raw = {1: torch.int8, 2: torch.int16, 4: torch.int32}[t.element_size()]
            assert torch.equal(t.view(raw), u.view(raw))


def test_calls_are_captured_and_replayed():
    c = Tree([(8, 300), (3, 90), (12, 700)], H=2, G=4, seed=72)
    w0 = weights_of(c)
    start = c.kv_len - (c.q_start[1:] - c.q_start[:-1])
    k0 = c.k.clone()

    def steps(w):
        out, lse = c.cache.attend(c.q, c.batch, lse=True)
        tr, _ = c.cache.attend(c.q, c.batch, tree=c.tree)
        c.cache.weigh(c.q, lse, c.batch, w)
        kept, count = c.cache.select(w, c.batch, 64, sinks=2, recent=8)
        c.cache.keep(kept, count, c.batch, weights=w)
        return out, tr, w, kept, count

    want = [t.clone() for t in steps(w0.clone())]
    k1 = c.k.clone()
    c.k.copy_(k0)
    w = w0.clone()
    v1 = c.v.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = steps(w)
    assert start.numel() == 3
    for _ in range(2):
        c.k.copy_(k0)
        w.copy_(w0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[3], want[3]) and torch.equal(got[4], want[4]) and torch.equal(got[2], want[2])
        assert torch.equal(c.k, k1)
        c.v.copy_(v1)
    assert c.cache.status() == R().LR_OK
