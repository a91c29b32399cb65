"""Attention over the paged cache at the edges of its range, with the bound of test_gpu_cache.py and no slack in it.

The terms of that bound that do not shrink with the values, derived for each product:
  16-bit caches   weights are rounded to the cache's type: fp16 ones below its normal range are off by 2^-25 each,
                  n 2^-25 V in all (n tokens, V = max |v|); an fp16 output is off by 2^-25 more
  8-bit caches    the weights' products are fp16 ones (single tokens, and chunks of an fp16 cache) or bf16 ones; what
                  an fp16 weight multiplies is at most V, or 2^-15 where V is below it (codes of up to 448 times
                  2^-24, the smallest power of two of fp16); such a product's own rounding is 2^-25 at most, once,
                  since the weights' sum is one
"""
import math

import pytest

torch = pytest.importorskip("torch")

import test_gpu_cache as base  # noqa: E402
from test_gpu_cache import C, DT, R, _built  # noqa: E402,F401

pytestmark = pytest.mark.gpu


class Case(base.Case):
    def reference(self, scale=None, window=0, sinks=0):
        out, lse, tol, ltol = super().reference(scale, window, sinks)
        t0 = 0
        for s, (ql, kv) in enumerate(self.seqs):
            rows = slice(t0, t0 + ql)
            t0 += ql
            if kv == 0 or ql == 0:
                continue
            for h in range(self.H):
                top = float(torch.nan_to_num(self.values("v", s, h, kv), 0.0, 0.0, 0.0).abs().max())
                slack = (kv + 1) * 2.0 ** -25 * (top + 1.0) if self.dt == "fp16" else 0.0
                mine = 0.0
                if self.fmt != "16":
                    mine = kv * 2.0 ** -25 * max(top, 2.0 ** -15) + (2.0 ** -24 if self.dt == "fp16" else 0.0)
                elif self.dt == "fp16":
                    mine = kv * 2.0 ** -25 * top + 2.0 ** -25
                tol[rows, h * self.G:(h + 1) * self.G] += mine - slack
        return out, lse, tol.clamp_(min=1e-30), ltol


@pytest.mark.parametrize("D,b", [(128, 16), (64, 32), (128, 5)])
@pytest.mark.parametrize("seqs,window,sinks", [([(1500, 1500), (2000, 2000)], 0, 0), ([(1000, 6000), (1048, 9000)], 1024, 4),
                                               ([(333, 333), (1111, 1111), (801, 2001)], 0, 0)])
def test_chunks_of_several_sequences(D, b, seqs, window, sinks):
    # CTAs that go from many tiles of a unit of at most 128 rows to a wider unit whose first tile has places of no token
    c = Case(seqs, H=8, G=4, D=D, b=b, seed=31, garbage=math.nan)
    a, la = c.check(window=window, sinks=sinks)
    for _ in range(3):
        x, lx = c.check(window=window, sinks=sinks)
        assert torch.equal(a, x) and torch.equal(la, lx)


STEPS = [(1, 3000), (2, 777), (1, 100)]   # at most 8 rows a sequence: the kernel of single tokens
CHUNKS = [(90, 2500), (300, 700)]         # more: the kernel of chunks


@pytest.mark.parametrize("seqs", [STEPS, CHUNKS], ids=["steps", "chunks"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("size", [1e-4, 1e-3, 1e-2, 30.0])
def test_values_of_any_size(seqs, dtype, fmt, size):
    c = Case(seqs, D=64, dtype=dtype, fmt=fmt, seed=32)
    if fmt == "16":
        c.v.mul_(size)
    else:
        c.v_scale.mul_(size)
    c.check()


@pytest.mark.parametrize("seqs", [STEPS, CHUNKS], ids=["steps", "chunks"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_values_of_mixed_sizes_and_signs(seqs, dtype, fmt):
    # a factor of 1e4 between tokens, and scales that a caller has made negative
    c = Case(seqs, D=64, dtype=dtype, fmt=fmt, seed=33)
    g = torch.Generator(device="cuda")
    g.manual_seed(34)
    c.v_scale.mul_(10.0 ** (4.0 * torch.rand(c.v_scale.shape, device="cuda", generator=g) - 3.0))
    c.check()
    c.v_scale.mul_(torch.where(torch.rand(c.v_scale.shape, device="cuda", generator=g) < 0.5, -1.0, 1.0))
    c.check()
    c.v_scale.copy_(-c.v_scale.abs())
    c.check()


@pytest.mark.parametrize("seqs", [STEPS, CHUNKS], ids=["steps", "chunks"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("scale", [2000.0, 20000.0])
def test_large_scales_of_small_codes(seqs, dtype, fmt, scale):
    # a caller's cache: code * scale is a number of either type, whatever the scale alone
    c = Case(seqs, D=64, dtype=dtype, fmt=fmt, seed=35)
    g = torch.Generator(device="cuda")
    g.manual_seed(36)
    codes = torch.randint(-2, 3, c.v.shape, device="cuda", generator=g)
    if fmt == "e4m3":
        c.v.view(torch.int8).copy_((codes.float() * 0.75).to(torch.float8_e4m3fn).view(torch.int8))
    else:
        c.v.copy_(codes.to(torch.int8))
    c.v_scale.fill_(scale)
    c.check()


@pytest.mark.parametrize("dtype,times", [("bf16", 1e7), ("fp16", 1e4)])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("ql,G", [(4, 2), (3, 5), (40, 4), (200, 2)])
def test_a_large_value_reaches_only_the_rows_that_see_it(dtype, times, fmt, ql, G):
    c = Case([(ql, 300)], H=2, G=G, D=64, dtype=dtype, fmt=fmt, seed=37)
    ref, _, tol, _ = c.reference()
    where = 300 - ql // 2
    c.v_scale[c.table[0, where // c.b].long(), where % c.b] *= times
    out = c.cache.attend(c.q, c.batch)[0].double()
    assert c.cache.status() == R().LR_OK
    hidden = ql - (300 - where)  # rows before it
    assert bool(((out - ref).abs() <= tol)[:hidden].all())
    assert bool(((out - ref).abs() > tol)[hidden:].any())


@pytest.mark.parametrize("dtype,times", [("bf16", 1e7), ("fp16", 1e4)])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_large_value_of_no_weight(dtype, times, fmt):
    # single tokens: fp16 weights are taken against the largest product of weight and scale, not the largest scale
    c = Case([(1, 300), (2, 80)], H=2, G=2, D=64, dtype=dtype, fmt=fmt, seed=38)
    c.q.abs_()
    blk, off = c.table[0, 5].long(), 7
    c.k.view(torch.int8)[blk, off] = torch.full((2, 64), -8.0).to(torch.float8_e4m3fn).view(torch.int8).cuda() if fmt == "e4m3" else -8
    c.k_scale[blk, off] = 10.0  # a score of about -80 * 1.2 * 64 / 8: its weight is nothing
    ref, _, tol, _ = c.reference()
    c.v_scale[blk, off] *= times
    out = c.cache.attend(c.q, c.batch)[0].double()
    assert c.cache.status() == R().LR_OK
    assert bool(((out - ref).abs() <= tol).all())


@pytest.mark.parametrize("fmt", ["16", "e4m3", "int8"])
@pytest.mark.parametrize("D,b", [(64, 16), (128, 5), (64, 1), (64, 64)])
@pytest.mark.parametrize("ql,kv,G,window,sinks,place", [(90, 300, 4, 0, 0, 295), (200, 300, 2, 0, 0, 150), (200, 300, 2, 40, 3, 130),
                                                        (150, 400, 4, 40, 3, 1), (4, 290, 2, 0, 0, 289), (8, 261, 2, 0, 0, 258),
                                                        (8, 261, 1, 5, 2, 250), (1, 300, 4, 0, 0, 70)])
def test_a_block_out_of_range_reaches_only_the_rows_that_read_it(fmt, D, b, ql, kv, G, window, sinks, place):
    c = Case([(ql, kv), (2, 50)], H=2, G=G, D=D, b=b, fmt=fmt, seed=39)
    ref, rl, tol, ltol = c.reference(window=window, sinks=sinks)
    c.table[0, place // b] = c.nb
    out, lse = c.cache.attend(c.q, c.batch, window=window, sinks=sinks, lse=True)
    at = torch.arange(kv - ql, kv, device="cuda")[:, None]
    j = torch.arange(place // b * b, min(kv, place // b * b + b), device="cuda")[None]
    see = j <= at
    if window:
        see &= (j > at - window) | (j < sinks)
    reads = torch.cat([see.any(1), torch.zeros(2, dtype=torch.bool, device="cuda")])
    assert c.cache.status() == (R().LR_EINVAL if reads.any() else R().LR_OK)
    assert torch.isnan(out[reads]).all() and torch.isnan(lse[reads]).all()
    assert bool(((out.double() - ref).abs() <= tol)[~reads].all()) and bool(((lse.double() - rl).abs() <= ltol)[~reads].all())


@pytest.mark.parametrize("many", [0, 1500])
@pytest.mark.parametrize("fmt", ["16", "int8"])
def test_a_token_that_two_sequences_claim_has_no_place(fmt, many):
    # q_start 0, 5, 3, 8: the first sequence has tokens 0-4, the third 3-7, the second none
    c = Case([(5, 20), (0, 9), (5, 30)] + [(0, 1)] * many, H=2, G=1, D=32, b=8, fmt=fmt, seed=40)
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = C().CacheBatch(torch.tensor([0, 5, 3, 8] + [8] * many, **i32), c.kv_len, c.table, 8)
    before = [t.clone() for t in (c.k, c.v)]
    x = torch.randn((8, 2, 32), device="cuda").to(torch.bfloat16)
    c.cache.write(x, x, batch)
    assert c.cache.status() == R().LR_EINVAL
    k, v = c.cache.read(batch, 8)
    assert c.cache.status() == R().LR_EINVAL
    place = {t: (0, 15 + t) for t in range(5)}           # token: (sequence, position)
    place.update({t: (2, 25 + t - 3) for t in range(5, 8)})
    for got, now, was in ((k, c.k, before[0]), (v, c.v, before[1])):
        changed = (now != was).any(-1).any(-1)
        if not many:  # (in larger batches one of the two may have them)
            assert torch.isnan(got[3:5]).all()
            mine = torch.zeros_like(changed)
            for t in (0, 1, 2, 5, 6, 7):
                s, p = place[t]
                mine[c.table[s, p // 8].long(), p % 8] = True
            assert not changed[~mine].any()
        want = x
        if fmt != "16":
            codes, sc = base.quantised(x.float(), fmt)
            want = (codes.float() * sc[..., None]).to(torch.bfloat16)
        for t in (0, 1, 2, 5, 6, 7):
            assert torch.equal(got[t], want[t])


def test_numbers_beyond_32_bits_are_refused():
    # not taken modulo 2^32, where they could be others' valid ones
    c = Case([(2, 30), (1, 20)], H=2, G=4, D=64, seed=41)
    far = 1 << 32
    for kw in (dict(window=far), dict(window=far + 5), dict(window=-far + 5), dict(window=3, sinks=far + 1)):
        with pytest.raises(R().LRError) as e:
            c.cache.attend(c.q, c.batch, **kw)
        assert e.value.code == R().LR_EINVAL
    for max_q in (far + 2, -far + 2):
        with pytest.raises(R().LRError) as e:
            c.cache.attend(c.q, C().CacheBatch(c.q_start, c.kv_len, c.table, max_q))
        assert e.value.code == R().LR_EINVAL
    for kw in (dict(num_q_heads=far + 8), dict(max_seqs=far + 1)):
        with pytest.raises(R().LRError) as e:
            C().PagedCache(**{**dict(k=c.k, v=c.v, num_q_heads=8), **kw})
        assert e.value.code == R().LR_EINVAL


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("size", [1e-5, 1e-4, 3e-4, 1e-3, 1e-2])
def test_rows_that_see_one_small_value(fmt, size):
    # a window of one token: the output is its V, and nothing averages what the product rounds
    c = Case([(300, 300), (200, 900)], H=2, G=2, D=64, dtype="fp16", fmt=fmt, seed=42)
    c.v_scale.mul_(size)
    c.check(window=1)
