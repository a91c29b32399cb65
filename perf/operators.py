"""Performance cases of the paged KV cache and its attention, through their Python entry points.

A serving engine executes the batches that the router's simulation counts: each batch brings the
last tokens of a set of sequences (one token of a sequence that decodes, a chunk of one in
prefill), stores their K and V in a paged cache and attends over it.  Three operators:

  store    the new tokens' K and V are quantised (or kept) as they are written into their
           blocks, and the same tokens are read back as values
  load     whole sequences are read back from the cache (a sequence handed to another instance)
  attend   attention of the new tokens over the cached ones, causal, optionally with a
           sliding window and a few first tokens that stay visible

Sizes follow the repository's workloads (token budgets of 2,048 to 8,192, 64 and 256 sequences, blocks
of 16 tokens, prompts up to 32,768 tokens), and odd sizes between and around them.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------
# The cases

BASE = {"singles": 0, "chunks": 0, "chunk_tokens": 0, "ctx_lo": 1, "ctx_hi": 1, "q_heads": 32, "kv_heads": 8,
        "head_dim": 128, "block": 16, "dtype": "bf16", "fmt": "16", "heads_first": False, "fused": False,
        "window": 0, "sinks": 0, "lse": False}
STORE = dict(BASE, kind="store")
LOAD = dict(BASE, kind="load")
ATTEND = dict(BASE, kind="attend")


def listed():
    return [
        # one decode step of 64 sequences: 64 tokens into 64 blocks, where latency counts
        dict(STORE, name="store_step64", singles=64, ctx_lo=128, ctx_hi=8192, fmt="e4m3"),
        # one full token budget: two chunks beside 61 decoding sequences, K and V as slices of a fused projection
        dict(STORE, name="store_budget8192", singles=61, chunks=2, chunk_tokens=8131, ctx_lo=128, ctx_hi=8192, fmt="int8",
             fused=True),
        # whole prompts of a pool taken in at once, kept in 16 bits, blocks laid out by head
        dict(STORE, name="store_prompts", chunks=5, chunk_tokens=65000, ctx_lo=32768, ctx_hi=32768, dtype="fp16",
             block=32, heads_first=True),
        # one short sequence handed to another instance: heads of 96
        dict(LOAD, name="load_one", chunks=1, ctx_lo=1777, ctx_hi=1777, kv_heads=4, q_heads=16, head_dim=96, fmt="e4m3"),
        # an instance's 64 sequences moved at once
        dict(LOAD, name="load_pool64", chunks=64, ctx_lo=1024, ctx_hi=32768, fmt="int8", dtype="fp16"),
        # a single sequence's next token: the smallest call
        dict(ATTEND, name="step_one", singles=1, ctx_lo=1339, ctx_hi=1339, lse=True),
        # a decode step of 64 sequences over an 8-bit cache
        dict(ATTEND, name="step_64", singles=64, ctx_lo=128, ctx_hi=8192, fmt="e4m3"),
        # a decode step of 256 sequences that see a window and four first tokens
        dict(ATTEND, name="step_256_window", singles=256, ctx_lo=1024, ctx_hi=32768, fmt="int8", dtype="fp16", q_heads=64,
             window=1024, sinks=4),
        # one very long context: few rows, a long axis
        dict(ATTEND, name="step_long", singles=1, ctx_lo=200001, ctx_hi=200001, q_heads=24, kv_heads=4, heads_first=True),
        # a mixed batch of 2,048 tokens: 63 decoding sequences and a chunk
        dict(ATTEND, name="mixed_2048", singles=63, chunks=1, chunk_tokens=1985, ctx_lo=512, ctx_hi=6001, fused=True),
        # half a budget of new tokens at the end of the longest prompt: matrix products bound it
        dict(ATTEND, name="chunk_4096_long", chunks=1, chunk_tokens=4096, ctx_lo=32768, ctx_hi=32768),
        # two chunks under a window over an 8-bit cache, heads of 64
        dict(ATTEND, name="chunk_window", chunks=2, chunk_tokens=8001, ctx_lo=9000, ctx_hi=16001, q_heads=64, kv_heads=8,
             head_dim=64, block=64, fmt="e4m3", dtype="fp16", window=1024, sinks=4, lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(BASE, kind=rng.choice(["store", "load", "attend", "attend", "attend"]))
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 6, 8])
    c["head_dim"] = rng.choice([64, 64, 80, 96, 128, 128, 128])
    c["block"] = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 128])
    c["dtype"] = rng.choice(["bf16", "fp16"])
    c["fmt"] = rng.choice(["16", "e4m3", "int8"])
    c["heads_first"] = rng.random() < 0.3
    c["fused"] = rng.random() < 0.3
    c["ctx_lo"] = _log(rng, 1, 4096)
    c["ctx_hi"] = c["ctx_lo"] + _log(rng, 1, 28000)
    if c["kind"] == "store":
        c["singles"] = rng.choice([0, _log(rng, 1, 256)])
        c["chunks"] = rng.randint(0 if c["singles"] else 1, 4)
        c["chunk_tokens"] = _log(rng, max(1, c["chunks"]), 20000) if c["chunks"] else 0
    elif c["kind"] == "load":
        c["chunks"] = _log(rng, 1, 48)
    else:
        form = rng.choice(["singles", "chunks", "mixed"])
        if form != "chunks":
            c["singles"] = _log(rng, 1, 128)
        if form != "singles":
            c["chunks"] = rng.randint(1, 3)
            c["chunk_tokens"] = _log(rng, c["chunks"], 3000)
        if rng.random() < 0.4:
            c["window"] = _log(rng, 16, 4096)
            c["sinks"] = rng.choice([0, 1, 4, 16])
        c["lse"] = rng.random() < 0.5
    return c


# ---------------------------------------------------------------------------------------------
# Inputs

def _lengths(case):
    """(q_len, kv_len) of every sequence, from the case alone: contexts spread evenly over the logarithm
    of their range, the chunks' tokens in unequal parts, the decoding sequences first."""
    n = case["singles"] + case["chunks"]
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    ctx = [min(hi, max(1, round(lo * (hi / lo) ** ((i * 0.6180339887 + 0.5) % 1.0)))) for i in range(n)]
    q = [1] * case["singles"]
    if case["kind"] == "load":
        return ctx, ctx
    left, parts = case["chunk_tokens"], case["chunks"]
    for i in range(parts):
        mine = left if i == parts - 1 else max(1, min(left - (parts - 1 - i), round(left / (parts - i) * (0.7 if i % 2 else 1.2))))
        q.append(mine)
        left -= mine
    return q, [max(a, b) for a, b in zip(q, ctx)]


def _spread(case, g, *shape):
    """Activations: normal, with a few channels several times as large as the others."""
    x = torch.randn(*shape, device="cuda", dtype=torch.float32, generator=g)
    x[..., 3::37] *= 4.0
    return x


def _quantised(x, fmt):
    """(codes in their own type, scale) of fp32 vectors x [..., D]."""
    top = 448.0 if fmt == "e4m3" else 127.0
    a = x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100)
    y = x * (torch.full_like(a, top) / a)
    y = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().clamp(-127.0, 127.0).to(torch.int8)
    return y, (a / torch.full_like(a, top)).squeeze(-1)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q_len, kv_len = _lengths(case)
    n, H, D, b, dt = len(q_len), case["kv_heads"], case["head_dim"], case["block"], DTYPES[case["dtype"]]
    blocks = [-(-x // b) for x in kv_len]
    total = sum(blocks) + 7
    order = torch.randperm(total, device="cuda", generator=g, dtype=torch.int64).to(torch.int32)
    table = torch.zeros((n, max(blocks)), dtype=torch.int32, device="cuda")
    used = torch.arange(max(blocks), device="cuda")[None, :] < torch.tensor(blocks, device="cuda")[:, None]
    table[used] = order[:sum(blocks)]
    s = {"q_len": q_len, "kv_len_host": kv_len, "table": table, "max_q": max(q_len), "tokens": sum(q_len)}
    s["q_start"] = torch.tensor([0] + q_len, device="cuda").cumsum(0).to(torch.int32)
    s["kv_len"] = torch.tensor(kv_len, device="cuda", dtype=torch.int32)
    shape = (total, H, b, D) if case["heads_first"] else (total, b, H, D)
    for name in ("k", "v"):
        store = torch.empty(shape, device="cuda", dtype=dt if case["fmt"] == "16" else torch.float8_e4m3fn if case["fmt"] == "e4m3" else torch.int8)
        scale = None if case["fmt"] == "16" else torch.empty(shape[:3], device="cuda", dtype=torch.float32)
        step = max(1, (1 << 27) // (H * b * D))
        for i in range(0, total, step):  # in pieces: the fp32 values take four times the cache's room
            x = _spread(case, g, min(step, total - i), *shape[1:]).to(dt)
            if scale is None:
                store[i:i + step] = x
            else:
                codes, sc = _quantised(x.float(), case["fmt"])
                store[i:i + step], scale[i:i + step] = codes, sc
        s[name] = store.transpose(1, 2) if case["heads_first"] else store  # [block, token, head, D]
        s[name + "_scale"] = None if scale is None else scale.transpose(1, 2) if case["heads_first"] else scale
    T, Hq = s["tokens"], case["q_heads"]
    if case["kind"] == "store":
        if case["fused"]:
            x = _spread(case, g, T, Hq + 2 * H, D).to(dt)
            s["k_new"], s["v_new"] = x[:, Hq:Hq + H], x[:, Hq + H:]
        else:
            s["k_new"], s["v_new"] = _spread(case, g, T, H, D).to(dt), _spread(case, g, T, H, D).to(dt)
    if case["kind"] == "attend":
        x = _spread(case, g, T, Hq + (2 * H if case["fused"] else 0), D).to(dt)
        s["q"] = x[:, :Hq]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:  # the handle and the batch description that an engine keeps
        from paper_2607_18253_gb300 import cache as C
        s["cache"] = C.PagedCache(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], num_q_heads=case["q_heads"],
                                  dtype=DTYPES[case["dtype"]], max_seqs=len(s["q_len"]))
        s["batch"] = C.CacheBatch(s["q_start"], s["kv_len"], s["table"], s["max_q"])
    return s


# ---------------------------------------------------------------------------------------------
# One pass

def run(s):
    c = s["case"]
    if own:
        if c["kind"] == "attend":
            out, lse = s["cache"].attend(s["q"], s["batch"], window=c["window"], sinks=c["sinks"], lse=c["lse"])
            return {"out": out, "lse": lse} if c["lse"] else {"out": out}
        if c["kind"] == "store":
            s["cache"].write(s["k_new"], s["v_new"], s["batch"])
        k, v = s["cache"].read(s["batch"], s["tokens"])
        return _stored(s, k, v)
    if c["kind"] == "attend":
        return _attend(s, c)
    place = _places(s)
    if c["kind"] == "store":
        for name in ("k", "v"):
            x = s[name + "_new"]
            if c["fmt"] == "16":
                s[name][place] = x
            else:
                codes, scale = _quantised(x.float(), c["fmt"])
                s[name].view(torch.int8)[place] = codes.view(torch.int8)
                s[name + "_scale"][place] = scale
    return _stored(s, *(_values(s, name, *place).to(DTYPES[c["dtype"]]) for name in ("k", "v")))


def _stored(s, k, v):
    """What a store or load returns: the values read back; a store also the cache as it stands now."""
    if s["case"]["kind"] == "load":
        return {"k": k, "v": v}
    return {"k": k, "v": v, **{n: s[m] for n, m in (("k_cache", "k"), ("v_cache", "v"), ("k_scale", "k_scale"), ("v_scale", "v_scale"))}}


def _places(s):
    """(block, place in the block) of every token of the batch."""
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["q_start"], t, right=True, out_int32=True) - 1
    pos = s["kv_len"][seq] - s["q_start"][seq + 1] + t
    b = s["k"].shape[1]
    return s["table"][seq, pos // b].long(), pos % b


def _values(s, name, block, place):
    """fp32 values of the cached vectors at (block, place): [..., heads, D]."""
    if s[name + "_scale"] is None:
        return s[name][block, place].float()
    x = s[name].view(torch.int8)[block, place].view(s[name].dtype)
    return x.float() * s[name + "_scale"][block, place].unsqueeze(-1)


def _attend(s, c):
    T, Hq, D = s["tokens"], c["q_heads"], c["head_dim"]
    out = torch.empty((T, Hq, D), dtype=DTYPES[c["dtype"]], device="cuda")
    lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
    if c["singles"]:
        _padded(s, c, 0, c["singles"], out, lse)
    if c["chunks"]:
        _padded(s, c, c["singles"], c["singles"] + c["chunks"], out, lse)
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def _padded(s, c, first, last, out, lse):
    """Sequences first..last-1 as one dense, padded batch: products, a masked softmax, products."""
    n, H, D, b = last - first, c["kv_heads"], c["head_dim"], c["block"]
    Q, G = max(s["q_len"][first:last]), c["q_heads"] // c["kv_heads"]
    q_start, kv_len = s["q_start"][first:last].long(), s["kv_len"][first:last].long()
    q_len = s["q_start"][first + 1:last + 1].long() - q_start
    row = torch.arange(Q, device="cuda")[None, :]
    token = (q_start[:, None] + row).clamp(max=s["tokens"] - 1)
    at = kv_len[:, None] - q_len[:, None] + row                                     # the rows' positions [n, Q]
    # the cached tokens that some row of the sequence can see: the sinks, then from the first row's window on
    longest, window, sinks = max(s["kv_len_host"][first:last]), c["window"], c["sinks"] if c["window"] else 0
    start = (kv_len - q_len + 1 - window).clamp(min=sinks) if window else torch.zeros_like(kv_len)
    seen = min(longest, window + Q - 1) if window else longest
    pos = torch.cat([torch.arange(sinks, device="cuda").expand(n, sinks), start[:, None] + torch.arange(seen, device="cuda")], 1)
    real = pos < kv_len[:, None]
    pos = pos.clamp(max=longest - 1)
    block = s["table"][first:last].long().gather(1, pos // b)
    q = s["q"][token].float().view(n, Q, H, G, D).permute(0, 2, 3, 1, 4).reshape(n, H, G * Q, D)
    k = _values(s, "k", block, pos % b).transpose(1, 2)                              # [n, H, P, D]
    v = _values(s, "v", block, pos % b).transpose(1, 2)
    k, v = k.masked_fill(~real[:, None, :, None], 0.0), v.masked_fill(~real[:, None, :, None], 0.0)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).view(n, H, G, Q, -1)
    see = real[:, None, :] & (pos[:, None, :] <= at[:, :, None])
    if window:
        see &= (pos[:, None, :] > at[:, :, None] - window) | (pos[:, None, :] < sinks)
    p.masked_fill_(~see[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True).clamp(min=-3.0e38)
    p = p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, H, G * Q, -1), v).view(n, H, G, Q, D) / total.clamp(min=1e-30)
    l = torch.where(total > 0, m + total.log(), torch.full_like(m, -math.inf)).squeeze(-1)
    if Q == 1:
        out[first:last], lse[first:last] = o.reshape(n, H * G, D).to(out.dtype), l.reshape(n, H * G)
    else:
        keep = row < q_len[:, None]
        out[token[keep]] = o.permute(0, 3, 1, 2, 4).reshape(n, Q, H * G, D)[keep].to(out.dtype)
        lse[token[keep]] = l.permute(0, 3, 1, 2).reshape(n, Q, H * G)[keep]


# ---------------------------------------------------------------------------------------------
# Work and 64-bit values

def _seen(case):
    """(cached tokens that some row sees, visible (row, token) pairs) over the sequences, for one head."""
    w, sinks = case["window"], case["sinks"]
    tokens = pairs = 0
    for q, kv in zip(*_lengths(case)):
        first = kv - q
        if not w:
            tokens += kv
            pairs += q * first + q * (q + 1) // 2
            continue
        lo = max(0, first + 1 - w)
        tokens += kv - lo + min(sinks, lo)
        pairs += sum(min(i + 1, w) + min(sinks, max(0, i + 1 - w)) for i in range(first, kv))
    return tokens, pairs


def work(case):
    H, D = case["kv_heads"], case["head_dim"]
    cached = 2 * H * (D * 2 if case["fmt"] == "16" else D + 4)  # a token's K and V in the cache
    values = 2 * H * D * 2                                      # and as 16-bit values
    T = sum(_lengths(case)[0])
    if case["kind"] == "store":  # in, to the cache, and out again as values
        return {"bytes": T * (2 * values + cached), "flops": 0}
    if case["kind"] == "load":
        return {"bytes": T * (values + cached), "flops": 0}
    tokens, pairs = _seen(case)
    rows = T * case["q_heads"]
    return {"bytes": tokens * cached + rows * (4 * D + (4 if case["lse"] else 0)), "flops": 4 * D * pairs * case["q_heads"]}


def exact(case, seed):
    s = _inputs(case, seed)
    q_len, kv_len = s["q_len"], s["kv_len_host"]
    b, H, G, D = case["block"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]

    def cached(name, i, head, lo, hi):
        p = torch.arange(lo, hi, device="cuda")
        blk = s["table"][i].long()[p // b]
        x = s[name][:, :, head].view(torch.int8)[blk, p % b].view(s[name].dtype).double() if case["fmt"] != "16" else s[name][blk, p % b, head].double()
        return x if case["fmt"] == "16" else x * s[name + "_scale"][blk, p % b, head].double()[:, None]

    if case["kind"] == "load":
        return {n: torch.cat([torch.stack([cached(n, i, h, 0, kv) for h in range(H)], 1) for i, kv in enumerate(kv_len)]) for n in ("k", "v")}
    if case["kind"] == "store":
        got = {"k_cache": None, "v_cache": None, "k_scale": None, "v_scale": None}
        for n in ("k", "v"):
            x = s[n + "_new"].double()
            if case["fmt"] != "16":
                step = x.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100) / (448 if case["fmt"] == "e4m3" else 127)
                y = x / step
                if case["fmt"] == "e4m3":  # three bits after the leading one, the least exponent -6
                    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                    y = (y / ulp).round() * ulp
                else:
                    y = y.round()
                x = y * step
            got[n] = x
        return got
    out = torch.zeros((s["tokens"], H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], H * G), -math.inf, dtype=torch.float64, device="cuda")
    w, sinks, t0 = case["window"], case["sinks"], 0
    for i, (q, kv) in enumerate(zip(q_len, kv_len)):
        for h in range(H):
            k, v = cached("k", i, h, 0, kv), cached("v", i, h, 0, kv)
            for r in range(0, q, 2048):
                at = torch.arange(kv - q + r, kv - q + min(q, r + 2048), device="cuda")
                j = torch.arange(kv, device="cuda")[None, :]
                hide = j > at[:, None]
                if w:
                    hide |= (j <= at[:, None] - w) & (j >= sinks)
                rows = slice(t0 + r, t0 + r + len(at))
                z = torch.einsum("tgd,jd->tgj", s["q"][rows, h * G:(h + 1) * G].double(), k) / math.sqrt(D)
                z.masked_fill_(hide[:, None, :], -math.inf)
                l = torch.logsumexp(z, -1)
                out[rows, h * G:(h + 1) * G] = torch.exp(z - l[..., None]) @ v
                lse[rows, h * G:(h + 1) * G] = l
        t0 += q
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
