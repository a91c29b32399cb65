"""Trees and weights of cached tokens where their kernels can go wrong: tiles with columns of no row, infinities in lse and K, blocks
behind a window that are gone, groups of more heads than a tile has rows, an accepted path that is weighed.

A weight's comparison fails for a NaN.  The reference and the bound are those of test_gpu_cache_tokens.py: |w - want| <= tol in 64 bits, and places that no call
writes equal to the last bit (their bound is zero).
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_cache as base  # noqa: E402
from test_gpu_cache import C, R, SEQS, _built  # noqa: E402,F401
from test_gpu_cache_tokens import Tree, expected, weights_of  # noqa: E402

pytestmark = pytest.mark.gpu


def weighed(c, decay=1.0, window=0, sinks=0, scale=None, lse=None):
    """The call's weights, within their bound: every one of them a number."""
    w0 = weights_of(c)
    if lse is None:
        _, lse = c.cache.attend(c.q, c.batch, lse=True, window=window, sinks=sinks, scale=scale)
    w = c.cache.weigh(c.q, lse, c.batch, w0.clone(), decay=decay, window=window, sinks=sinks, scale=scale)
    assert c.cache.status() == R().LR_OK
    want, tol = expected(c, lse, w0, decay, window, sinks, scale)
    assert torch.isfinite(want).all() and torch.isfinite(tol).all()
    inside = (w.double() - want).abs() <= tol  # (false for a NaN)
    assert inside.all(), (int((~inside).sum()), int(torch.isnan(w).sum()))
    return w


# A sequence of several tiles of rows, full ones and a rest, a single token, and one whose rows are a tile and a few more (G = 3).
CHUNKS = [(130, 420), (1, 77), (43, 43), (86, 300)]
FORMS = [("16", "bf16", 16), ("16", "fp16", 5), ("e4m3", "bf16", 16), ("int8", "fp16", 24)]


@pytest.mark.parametrize("G", [3, 5, 6, 7, 40])
@pytest.mark.parametrize("D", [16, 64, 80, 96, 112, 128])
def test_weigh_tiles_with_columns_of_no_row(G, D):
    # G does not divide the 128 columns of a tile; scales on either side of where log2(e) times them is rounded to
    for fmt, dtype, b in FORMS:
        c = base.Case(CHUNKS, H=2, G=G, D=D, b=b, dtype=dtype, fmt=fmt, seed=80)
        for scale in (None, 1.0, 0.125, 0.11, 0.1):
            weighed(c, 0.5, scale=scale)
        for decay, window, sinks in ((1.0, 100, 4), (0.5, 100, 4), (0.5, 33, 0), (0.0, 1 << 20, 0)):
            weighed(c, decay, window, sinks)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seqs", list(SEQS))
def test_weigh_every_weight_is_a_number(fmt, dtype, seqs):
    for G, D, b in ((4, 128, 16), (1, 64, 1), (3, 80, 5), (8, 16, 16), (16, 96, 24), (17, 128, 64), (40, 64, 128)):
        c = base.Case(SEQS[seqs], G=G, D=D, b=b, dtype=dtype, fmt=fmt, seed=81)
        for decay in (1.0, 0.0, 0.9375):
            weighed(c, decay)
        weighed(c, 0.25, window=64, sinks=200)
        weighed(c, 1.0, window=17, sinks=3)
        weighed(c, 0.5, scale=0.7)


@pytest.mark.parametrize("G,D", [(3, 64), (7, 128), (4, 128)])
def test_weigh_infinite_keys(G, D):
    # a token that all rows see with a score of -inf receives nothing, and the others what they do without it
    c = base.Case([(130, 420)], H=1, G=G, D=D, seed=82)
    c.q[..., 5] = c.q[..., 5].abs() + 0.5
    blk, place = int(c.table[0, 2]), 7  # token 39
    c.k[blk, place] = 0.0
    _, lse = c.cache.attend(c.q, c.batch, lse=True)
    w0 = weights_of(c)
    want = c.cache.weigh(c.q, lse, c.batch, w0.clone(), decay=0.5)
    want[blk, place] = 0.5 * w0[blk, place]
    c.k[blk, place, :, 5] = -math.inf
    w = c.cache.weigh(c.q, lse, c.batch, w0.clone(), decay=0.5)
    assert c.cache.status() == R().LR_OK
    assert torch.isfinite(want).all() and torch.equal(w, want)


@pytest.mark.parametrize("fmt", ["16", "e4m3"])
@pytest.mark.parametrize("G,D", [(4, 128), (4, 64), (3, 80), (4, 112), (16, 64)])
def test_rows_of_infinite_lse_add_nothing(fmt, G, D):
    # exp(x - inf) is zero, whichever sign the rest of log2(e)'s rounding has; single rows, some of a tile, a tile's all
    for seqs in ([(1, 300), (2, 90)], [(130, 420), (1, 77)]):
        c = base.Case(seqs, G=G, D=D, fmt=fmt, seed=83)
        _, lse = c.cache.attend(c.q, c.batch, lse=True)
        for value in (math.inf, -math.inf):
            l = lse.clone()
            l[0], l[-1] = value, value
            weighed(c, 0.5, lse=l)
            l[::3] = value
            weighed(c, 1.0, lse=l)
            l[:, 1:] = value
            weighed(c, 0.0, lse=l)
        mixed = lse.clone()
        mixed[::2], mixed[1::4] = math.inf, -math.inf
        weighed(c, 0.5, lse=mixed)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("G,D,b", [(20, 112, 3), (4, 128, 16), (6, 64, 16), (12, 80, 8)])
def test_weigh_short_sequences_before_long_ones(fmt, G, D, b):
    # runs of units of at most 128 tokens, which half of a CTA's warps skip, before units of 256, many of each a CTA
    seqs = [s for i in range(40) for s in [(12, 12 + (7 * i + j) % 110) for j in range(1 + i % 9)] + [(11 + i % 90, 2000 + 331 * i)]]
    c = base.Case(seqs, H=2, G=G, D=D, b=b, fmt=fmt, seed=90)
    for decay, window, sinks in ((0.5, 0, 0), (0.5, 1, 16), (1.0, 700, 4)):
        a = weighed(c, decay, window, sinks)
        assert torch.equal(a, weighed(c, decay, window, sinks))
    d = base.Case([(2, 2), (11, 19649), (101, 31713), (2, 16)], H=3, G=G, D=D, b=b, fmt=fmt, seed=91)
    for decay, window, sinks in ((0.5, 1, 16), (0.0, 0, 0)):
        weighed(d, decay, window, sinks)


# ---------------------------------------------------------------------------------------------
# trees under a window: blocks that no row reads any more

def gone(c, window, sinks):
    """A block table without the blocks whose tokens no row of a chain or tree that names itself sees: those at or below context - window."""
    table = c.table.clone()
    for s, (ql, kv) in enumerate(c.seqs):
        lowest = kv - ql - window + 1  # the root's first token
        for i in range(max(0, lowest) // c.b):
            if i * c.b >= sinks:
                table[s, i] = -1
    return table


@pytest.mark.parametrize("fmt,b", [("16", 16), ("16", 5), ("16", 1), ("e4m3", 16), ("int8", 7)])
@pytest.mark.parametrize("sinks", [0, 4])
def test_tree_blocks_behind_the_window_may_be_gone(fmt, b, sinks):
    # contexts whose last hidden token ends a block, and others; few rows, many, and a unit of several CTAs
    for seqs, G in (([(4, 4 + 96), (1, 1 + 111), (2, 2 + 64), (3, 200)], 2), ([(40, 40 + 320), (64, 64 + 35), (7, 7 + 175)], 4),
                    ([(16, 16 + 40000)], 4)):
        for window in (32, 35):
            c = Tree(seqs, G=G, b=b, fmt=fmt, seed=84)
            want, wl = c.cache.attend(c.q, c.batch, window=window, sinks=sinks, lse=True, tree=c.tree)
            assert c.cache.status() == R().LR_OK
            batch = C().CacheBatch(c.q_start, c.kv_len, gone(c, window, sinks), max(q for q, _ in seqs))
            out, lse = c.cache.attend(c.q, batch, window=window, sinks=sinks, lse=True, tree=c.tree)
            assert c.cache.status() == R().LR_OK, window
            assert torch.isfinite(want).all() and torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.parametrize("fmt,b", [("16", 16), ("16", 5), ("e4m3", 16), ("int8", 7)])
@pytest.mark.parametrize("q,G", [(4, 2), (40, 4)])
def test_tree_rows_that_read_a_block_that_is_gone(fmt, b, q, G):
    # a row that names nothing stands at the context's last position and sees one token more than the others: where its block is gone,
    # that row alone is NaN, and the error recorded
    window = 32
    c = Tree([(q, q + window + 3 * b - 1), (q, q + 200)], G=G, b=b, fmt=fmt, seed=85)
    table = c.table.clone()
    table[0, :3] = c.nb  # tokens below context - window + 1
    batch = C().CacheBatch(c.q_start, c.kv_len, table, q)
    want, _ = c.cache.attend(c.q, c.batch, window=window, tree=c.tree)
    out, _ = c.cache.attend(c.q, batch, window=window, tree=c.tree)
    assert c.cache.status() == R().LR_OK and torch.equal(out, want)
    masks = c.tree.clone()
    masks[1] = 0
    out, _ = c.cache.attend(c.q, batch, window=window, tree=masks)
    assert c.cache.status() == R().LR_EINVAL and c.cache.status() == R().LR_OK
    assert torch.isnan(out[1]).all()
    assert torch.equal(torch.cat([out[:1], out[2:]]), torch.cat([want[:1], want[2:]]))


# ---------------------------------------------------------------------------------------------
# calls together, and the widest groups

@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("G,D", [(65, 64), (130, 16), (256, 64), (1024, 16)])
def test_groups_of_more_heads_than_a_tile_has_rows(fmt, G, D):
    for seqs in ([(1, 300), (2, 40)], [(5, 290), (1, 1), (3, 3)]):
        c = Tree(seqs, H=1, G=G, D=D, fmt=fmt, seed=86)
        c.check()
        c.check(window=33, sinks=2)
        for decay, window in ((1.0, 0), (0.5, 40)):
            weighed(base.Case(seqs, H=1, G=G, D=D, fmt=fmt, seed=87), decay, window, 2)


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 3)])
def test_a_chain_is_the_causal_call(fmt, window, sinks):
    # within the causal reference's own bounds, over 8 bits as well
    for seqs in ([(4, 40), (16, 16), (1, 33)], [(70, 900), (33, 161)]):
        c = Tree(seqs, fmt=fmt, seed=88)
        rows = [np.packbits(np.tril(np.ones((q, c.words * 32), bool)), axis=1, bitorder="little").view(np.int32) for q, _ in seqs]
        chain = torch.from_numpy(np.concatenate(rows)).cuda()
        want, wl, tol, ltol = base.Case.reference(c, None, window, sinks)
        out, lse = c.cache.attend(c.q, c.batch, window=window, sinks=sinks, lse=True, tree=chain)
        assert c.cache.status() == R().LR_OK
        assert bool(((out.double() - want).abs() <= tol).all()) and bool(((lse.double() - wl).abs() <= ltol).all())


@pytest.mark.parametrize("fmt", ["16", "int8"])
@pytest.mark.parametrize("seqs,G", [([(8, 100), (5, 37), (16, 16)], 2), ([(64, 300), (40, 90)], 3)])
def test_an_accepted_path_is_weighed(fmt, seqs, G):
    # a tree is verified and its deepest path moved up; the path's rows, gathered with the lse that the tree's attention gave, are
    # then the sequence's last causal ones
    c = Tree(seqs, H=2, G=G, D=64, fmt=fmt, seed=89)
    _, lse = c.check()
    lse = lse.float()
    rows, counts, starts = [], [], []
    kept = torch.full((len(seqs), max(q for q, _ in seqs)), -1, dtype=torch.int32, device="cuda")
    for s, (q, kv) in enumerate(seqs):
        path = torch.nonzero(c.paths[s][int(c.paths[s].sum(1).argmax())]).flatten()
        kept[s, :len(path)] = (kv - q + path).to(torch.int32)
        rows.append(int(c.q_start[s]) + path)
        counts.append(len(path))
        starts.append(kv - q)
    rows = torch.cat(rows)
    w0 = weights_of(c)
    c.cache.keep(kept, torch.tensor(counts, dtype=torch.int32, device="cuda"), c.batch, weights=w0,
                 start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    d = base.Case.__new__(base.Case)
    d.__dict__.update({k: v for k, v in c.__dict__.items()})
    d.seqs, d.T, d.q = [(n, a + n) for n, a in zip(counts, starts)], len(rows), c.q[rows].contiguous()
    d.q_start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    d.kv_len = torch.tensor([a + n for n, a in zip(counts, starts)], dtype=torch.int32, device="cuda")
    d.batch = C().CacheBatch(d.q_start, d.kv_len, d.table, max(counts))
    w = d.cache.weigh(d.q, lse[rows].contiguous(), d.batch, w0.clone(), decay=0.5)
    assert d.cache.status() == R().LR_OK
    want, tol = expected(d, lse[rows], w0, 0.5)
    assert bool(((w.double() - want).abs() <= tol).all())
    d.check()
