"""Performance cases of what an engine does with a paged KV cache beside storing and causal attention, through
the Python entry points of the cache.

  tree    attention of a tree of drafted tokens over the cache: a row sees the context and the drafted tokens that
          its mask names (speculative decoding verifies many continuations in one batch)
  weigh   the attention weight that the cached tokens have received, summed over a batch's rows
  evict   of every sequence and KV head the tokens with the largest weights are kept, beside the first and the most recent
          ones, and moved together, in place
  accept  the accepted path of a verified tree is moved up behind its context: the same move, by lists given

Sizes follow the repository's workloads (64 and 256 sequences, blocks of 16 tokens, prompts up to 32,768 tokens, chunks
of up to 4,096) and its cases of the cache's attention, and odd sizes between and around them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------
# The cases

BASE = {"seqs": 1, "q_lo": 1, "q_hi": 1, "ctx_lo": 1, "ctx_hi": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "block": 16,
        "dtype": "bf16", "fmt": "16", "heads_first": False, "window": 0, "sinks": 0}
TREE = dict(BASE, kind="tree", lse=False)
WEIGH = dict(BASE, kind="weigh", decay=1.0)
EVICT = dict(BASE, kind="evict", budget=1, share=0.0, recent=0)
ACCEPT = dict(BASE, kind="accept", path=1)


def listed():
    return [
        # one user's draft of eight tokens: the smallest verification, where latency counts
        dict(TREE, name="tree_one", q_lo=8, q_hi=8, ctx_lo=1339, ctx_hi=1339, lse=True),
        # a step of 64 sequences, each with a small tree, over an 8-bit cache
        dict(TREE, name="tree_64", seqs=64, q_lo=4, q_hi=16, ctx_lo=128, ctx_hi=8192, fmt="e4m3"),
        # a tree of 64 over one very long context
        dict(TREE, name="tree_long", q_lo=64, q_hi=64, ctx_lo=200001, ctx_hi=200001, q_heads=24, kv_heads=4, heads_first=True),
        # wide trees of an offline job, under a window and four first tokens, heads of 64, odd blocks
        dict(TREE, name="tree_wide", seqs=8, q_lo=201, q_hi=512, ctx_lo=1024, ctx_hi=16001, head_dim=64, q_heads=64, block=24,
             fmt="int8", dtype="fp16", window=1024, sinks=4, lse=True),
        # a decode step of 64 sequences adds its weights
        dict(WEIGH, name="weigh_step64", seqs=64, ctx_lo=128, ctx_hi=8192, fmt="e4m3"),
        # the last 32 tokens of five prompts weigh all of them, before the prompts are cut down
        dict(WEIGH, name="weigh_last32", seqs=5, q_lo=32, q_hi=32, ctx_lo=4096, ctx_hi=32768, decay=0.0),
        # a chunk at the end of the longest prompt: matrix products and exponentials bound it
        dict(WEIGH, name="weigh_chunk4096", q_lo=4096, q_hi=4096, ctx_lo=32768, ctx_hi=32768),
        # one short sequence cut down, heads of 96
        dict(EVICT, name="evict_one", ctx_lo=1777, ctx_hi=1777, q_heads=16, kv_heads=4, head_dim=96, fmt="e4m3", budget=512, recent=64,
             sinks=4),
        # an instance's 64 sequences cut down at once
        dict(EVICT, name="evict_pool64", seqs=64, ctx_lo=1024, ctx_hi=32768, fmt="int8", dtype="fp16", budget=2048, recent=256, sinks=4),
        # one very long context cut to a tenth
        dict(EVICT, name="evict_long", ctx_lo=200001, ctx_hi=200001, q_heads=24, kv_heads=4, heads_first=True, budget=20000, share=0.1,
             recent=1024, sinks=4),
        # the accepted paths of 64 small trees
        dict(ACCEPT, name="accept_64", seqs=64, q_lo=4, q_hi=16, ctx_lo=128, ctx_hi=8192, fmt="e4m3", path=4),
        # the accepted paths of 256 large ones
        dict(ACCEPT, name="accept_256", seqs=256, q_lo=32, q_hi=64, ctx_lo=128, ctx_hi=2048, path=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "weigh", "weigh", "evict", "accept"])
    c = dict({"tree": TREE, "weigh": WEIGH, "evict": EVICT, "accept": ACCEPT}[kind])
    c["kv_heads"] = rng.choice([1, 2, 4, 5, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 6, 8])
    c["head_dim"] = rng.choice([64, 64, 80, 96, 128, 128, 128])
    c["block"] = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 128])
    c["dtype"] = rng.choice(["bf16", "fp16"])
    c["fmt"] = rng.choice(["16", "e4m3", "int8"])
    c["heads_first"] = rng.random() < 0.3
    c["seqs"] = _log(rng, 1, 64)
    c["ctx_lo"] = _log(rng, 1, 4096)
    c["ctx_hi"] = c["ctx_lo"] + _log(rng, 1, 28000 if c["seqs"] <= 32 else 12000)
    if kind == "tree":
        c["q_lo"] = _log(rng, 1, 64)
        c["q_hi"] = c["q_lo"] + _log(rng, 1, 16 if c["seqs"] > 16 else 200)
        c["lse"] = rng.random() < 0.5
    if kind == "weigh":
        c["q_lo"] = c["q_hi"] = 1
        if rng.random() < 0.6:
            c["q_lo"] = _log(rng, 1, 64)
            c["q_hi"] = c["q_lo"] + _log(rng, 1, 64 if c["seqs"] > 8 else 1500)
        c["decay"] = rng.choice([1.0, 1.0, 0.0, 0.9375])
    if kind in ("tree", "weigh") and rng.random() < 0.4:
        c["window"] = _log(rng, 16, 4096)
        c["sinks"] = rng.choice([0, 1, 4, 16])
    if kind == "evict":
        c["sinks"], c["recent"] = rng.choice([0, 1, 4, 16]), rng.choice([0, 1, 32, 255])
        c["budget"] = c["sinks"] + c["recent"] + _log(rng, 1, 8192)
        c["share"] = rng.choice([0.0, 0.0, 0.2, 0.5])
    if kind == "accept":
        c["q_lo"] = _log(rng, 1, 64)
        c["q_hi"] = c["q_lo"] + _log(rng, 1, 64)
        c["path"] = _log(rng, 1, 20)
    return c


# ---------------------------------------------------------------------------------------------
# Inputs

def _lengths(case):
    """(q_len, kv_len) of every sequence, from the case alone: contexts spread evenly over the logarithm of their range,
    numbers of new tokens evenly over theirs."""
    n = case["seqs"]
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    ctx = [min(hi, max(1, round(lo * (hi / lo) ** ((i * 0.6180339887 + 0.5) % 1.0)))) for i in range(n)]
    q = [case["q_lo"] + round((case["q_hi"] - case["q_lo"]) * ((i * 0.7548776662 + 0.5) % 1.0)) for i in range(n)]
    if case["kind"] == "evict":
        return [1] * n, ctx
    return q, [max(a, b) for a, b in zip(q, ctx)]


def _budgets(case):
    """Tokens that each sequence may keep."""
    least = case["sinks"] + case["recent"]
    return [min(case["budget"], max(least, round(case["share"] * kv))) if case["share"] else case["budget"] for kv in _lengths(case)[1]]


def _paths(case):
    """Lengths of the accepted paths (the token after the context is always accepted)."""
    return [min(q, 1 + round((case["path"] - 1) * ((i * 0.5698402910 + 0.5) % 1.0))) for i, q in enumerate(_lengths(case)[0])]


def _spread(g, *shape):
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


def _trees(rng, q_len):
    """Masks of random trees, one bit a drafted token, 32 a word: the ancestors of each token and itself.  The
    first token is the root; a parent is more often a recent token than a far one."""
    most = max(q_len)
    words = -(-most // 32)
    n = len(q_len)
    see = np.zeros((n, most, words * 32), bool)
    for i in range(most):
        if i:
            back = np.minimum(i, 1 + rng.exponential(max(1.0, i / 3), n).astype(np.int64))
            see[:, i] = see[np.arange(n), i - back]
        see[:, i, i] = True
    bits = (see.reshape(n, most, words, 32).astype(np.uint32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint64).astype(np.uint32)
    return np.concatenate([bits[s, :q] for s, q in enumerate(q_len)]).view(np.int32)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
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
            x = _spread(g, min(step, total - i), *shape[1:]).to(dt)
            if scale is None:
                store[i:i + step] = x
            else:
                codes, sc = _quantised(x.float(), case["fmt"])
                store[i:i + step], scale[i:i + step] = codes, sc
        s[name] = store.transpose(1, 2) if case["heads_first"] else store  # [block, token, head, D]
        s[name + "_scale"] = None if scale is None else scale.transpose(1, 2) if case["heads_first"] else scale
    T, Hq = s["tokens"], case["q_heads"]
    if case["kind"] in ("tree", "weigh"):
        s["q"] = _spread(g, T, Hq, D).to(dt)
    if case["kind"] == "tree":
        s["tree"] = torch.from_numpy(_trees(rng, q_len)).cuda()
    if case["kind"] in ("weigh", "evict"):
        # accumulated weights: far apart, many of them small, the least of them equal
        w = torch.exp(2.0 * torch.randn(shape[:3], device="cuda", generator=g) - 2.0)
        w = torch.where(w < 0.03125, torch.floor(w * 512.0) / 512.0, w)
        s["weights"] = w.transpose(1, 2) if case["heads_first"] else w
    if case["kind"] == "evict":
        s["budget"] = torch.tensor(_budgets(case), dtype=torch.int32, device="cuda")
    if case["kind"] == "accept":
        paths = _paths(case)
        kept = np.full((n, max(paths)), -1, np.int32)
        for i, (q, kv, p) in enumerate(zip(q_len, kv_len, paths)):
            steps = np.sort(rng.permutation(np.arange(1, q))[:p - 1])
            kept[i, 0], kept[i, 1:p] = kv - q, kv - q + steps
        s["kept"] = torch.from_numpy(kept).cuda()
        s["count"] = torch.tensor(paths, dtype=torch.int32, device="cuda")
        s["start"] = s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "weigh":  # what the attention of these rows gave
        s["lse"] = torch.cat([x.logsumexp(-1).permute(0, 3, 1, 2).flatten(2)[keep] for x, keep, _ in _scores(s, case, by_rows=False)])
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
    if c["kind"] == "tree":
        if own:
            out, lse = s["cache"].attend(s["q"], s["batch"], window=c["window"], sinks=c["sinks"], lse=c["lse"], tree=s["tree"])
        else:
            out, lse = _attend(s, c)
        return {"out": out, "lse": lse} if c["lse"] else {"out": out}
    if c["kind"] == "weigh":
        if own:
            s["cache"].weigh(s["q"], s["lse"], s["batch"], s["weights"], decay=c["decay"], window=c["window"], sinks=c["sinks"])
        else:
            _weigh(s, c)
        return {"weights": s["weights"]}
    if c["kind"] == "evict":
        if own:
            kept, count = s["cache"].select(s["weights"], s["batch"], c["budget"], budget=s["budget"] if c["share"] else None,
                                            sinks=c["sinks"], recent=c["recent"])
            s["cache"].keep(kept, count, s["batch"], weights=s["weights"])
        else:
            kept, count = _select(s, c)
            _keep(s, kept, count, torch.zeros_like(count))
        return {"kept": kept, "count": count, "weights": s["weights"], **_cached(s)}
    if own:
        s["cache"].keep(s["kept"], s["count"], s["batch"], start=s["start"])
    else:
        _keep(s, s["kept"][:, None].expand(-1, c["kv_heads"], -1), s["count"], s["start"])
    return _cached(s)


def _cached(s):
    return {n: s[m] for n, m in (("k_cache", "k"), ("v_cache", "v"), ("k_scale", "k_scale"), ("v_scale", "v_scale")) if s[m] is not None}


def _values(s, name, block, place):
    """fp32 values of the cached vectors at (block, place): [..., heads, D]."""
    if s[name + "_scale"] is None:
        return s[name][block, place].float()
    x = s[name].view(torch.int8)[block, place].view(s[name].dtype)
    return x.float() * s[name + "_scale"][block, place].unsqueeze(-1)


def _tokens(s):
    """(positions, block, place) of all sequences' tokens, padded: [L], [n, L], [n, L]."""
    b, longest = s["k"].shape[1], max(s["kv_len_host"])
    pos = torch.arange(longest, device="cuda")
    return pos, s["table"].long()[:, pos // b], (pos % b).expand(len(s["q_len"]), longest)


def _seen(s, c, row):
    """Which tokens the rows `row` of every sequence see: [n, R, L]."""
    pos, _, _ = _tokens(s)
    q_len, kv_len = (s["q_start"][1:] - s["q_start"][:-1]).long()[:, None, None], s["kv_len"].long()[:, None, None]
    first, pos, row = kv_len - q_len, pos[None, None, :], row[None, :, None]
    window, sinks = c["window"], c["sinks"]
    if c["kind"] != "tree":
        at = first + row
        see = (pos <= at) & (pos >= 0)
        if window:
            see &= (pos > at - window) | (pos < sinks)
        return see & (row < q_len)
    token = (s["q_start"][:-1].long()[:, None] + row[0, :, 0]).clamp(max=s["tokens"] - 1)
    bits = s["tree"][token]                                                       # [n, R, words]
    i = (pos - first).clamp(min=0, max=32 * bits.shape[2] - 1)                     # drafted token, [n, 1, L]
    i = i.expand(-1, row.shape[1], -1)
    drafted = (bits.gather(2, i >> 5) >> (i & 31) & 1).bool() & (pos >= first) & (pos < kv_len)
    see = (pos < first).expand_as(drafted)
    if window:  # a drafted token's position is the context's length and how many drafted tokens come before it on its path
        depth = drafted.long().cumsum(2)
        at = first + depth[:, :, -1:] - 1
        place = torch.where(pos < first, pos, first + depth - 1)
        return ((see | drafted) & ((place > at - window) | (place < sinks))) & (row < q_len)
    return (see | drafted) & (row < q_len)


def _scores(s, c, by_rows=True):
    """Pieces of the masked scores of the padded batch: (scores [m, H, G, R, L], which (sequence, row) pairs are real [m, R],
    the piece's sequences and rows), by ranges of rows, or of sequences in turn (the rows' own order)."""
    H, D, n = c["kv_heads"], c["head_dim"], len(s["q_len"])
    Q, G = max(s["q_len"]), c["q_heads"] // c["kv_heads"]
    pos, block, place = _tokens(s)
    many = max(1, (1 << 32) // (c["q_heads"] * len(pos)))                          # (sequence, row) pairs of a piece
    pieces = [(0, n, r, min(Q, r + max(1, many // n))) for r in range(0, Q, max(1, many // n))] if by_rows else \
        [(i, i + 1, 0, Q) for i in range(n)] if many < n * Q else [(0, n, 0, Q)]
    for a, z, r0, r1 in pieces:
        k = _values(s, "k", block[a:z], place[a:z]).permute(0, 2, 3, 1)            # [m, H, D, L]
        row = torch.arange(r0, r1, device="cuda")
        q_start = s["q_start"].long()
        keep = row[None, :] < (q_start[a + 1:z + 1] - q_start[a:z])[:, None]
        token = (q_start[a:z, None] + row).clamp(max=s["tokens"] - 1)
        q = s["q"][token].float().view(z - a, r1 - r0, H, G, D).permute(0, 2, 3, 1, 4).reshape(z - a, H, -1, D)
        x = torch.matmul(q, k).mul_(D ** -0.5).view(z - a, H, G, r1 - r0, -1)
        x.masked_fill_(~_seen(s, c, row)[a:z, None, None], -math.inf)
        yield x, keep, (a, z, r0, r1)


def _attend(s, c):
    T, Hq, D, H = s["tokens"], c["q_heads"], c["head_dim"], c["kv_heads"]
    out = torch.empty((T, Hq, D), dtype=DTYPES[c["dtype"]], device="cuda")
    lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
    _, block, place = _tokens(s)
    for p, keep, (a, z, r0, r1) in _scores(s, c):
        v = _values(s, "v", block[a:z], place[a:z]).transpose(1, 2)                # [m, H, L, D]
        m = p.amax(-1, keepdim=True).clamp(min=-3.0e38)
        p = p.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(2, 3), v).view(*p.shape[:4], D) / total.clamp(min=1e-30)
        l = torch.where(total > 0, m + total.log(), torch.full_like(m, -math.inf)).squeeze(-1)
        token = (s["q_start"][a:z].long()[:, None] + torch.arange(r0, r1, device="cuda"))[keep]
        out[token] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[keep].to(out.dtype)
        lse[token] = l.permute(0, 3, 1, 2).flatten(2)[keep]
    return out, lse


def _weigh(s, c):
    H, G = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    pos, block, place = _tokens(s)
    total = torch.zeros((len(s["q_len"]), len(pos), H), device="cuda")
    for x, keep, (a, z, r0, r1) in _scores(s, c):
        token = (s["q_start"][a:z].long()[:, None] + torch.arange(r0, r1, device="cuda")).clamp(max=s["tokens"] - 1)
        l = s["lse"][token].view(z - a, r1 - r0, H, G).permute(0, 2, 3, 1).unsqueeze(-1)
        l = torch.where(l > -math.inf, l, torch.zeros_like(l))                     # (a row that sees nothing adds nothing)
        total[a:z] += x.sub_(l).exp_().sum((2, 3)).transpose(1, 2)
    kv_len, q_len = s["kv_len"].long()[:, None], (s["q_start"][1:] - s["q_start"][:-1]).long()[:, None]
    real, old = pos < kv_len, (pos < kv_len - q_len).unsqueeze(-1)
    w = s["weights"]
    if c["decay"]:
        total += torch.where(old, c["decay"] * w[block, place], torch.zeros_like(total))
    w[block[real], place[real]] = total[real]


def _select(s, c):
    n, H, cap = len(s["q_len"]), c["kv_heads"], c["budget"]
    pos, block, place = _tokens(s)
    kv_len = s["kv_len"].long()[:, None, None]
    w = s["weights"][block, place].transpose(1, 2)                                  # [n, H, L]
    # first tokens and recent ones come before all others; what is no token after
    must = (pos < c["sinks"]) | (pos >= kv_len - c["recent"])
    w = torch.where(must, torch.full_like(w, math.inf), w).masked_fill(pos >= kv_len, -math.inf)
    rank = torch.sort(w, dim=-1, descending=True, stable=True).indices
    count = torch.minimum(s["kv_len"], s["budget"])
    width = min(cap, len(pos))
    mine = torch.arange(width, device="cuda") < count[:, None, None]
    far = torch.full((1, 1, 1), 1 << 40, device="cuda")
    best = torch.sort(torch.where(mine, rank[:, :, :width], far), dim=-1).values
    kept = torch.full((n, H, cap), -1, dtype=torch.int32, device="cuda")
    kept[:, :, :width] = torch.where(mine, best, torch.full_like(far, -1)).to(torch.int32)
    return kept, count


def _keep(s, kept, count, start):
    """The tokens kept[sequence, head, i], i < count, moved to places start + i."""
    H, b = kept.shape[1], s["k"].shape[1]
    i = torch.arange(kept.shape[2], device="cuda")
    seq, head, nth = torch.nonzero((i < count[:, None, None]).expand_as(kept), as_tuple=True)
    src, dst = kept[seq, head, nth].long(), start[seq].long() + nth
    table = s["table"].long()
    src, dst = (table[seq, src // b], src % b, head), (table[seq, dst // b], dst % b, head)
    for name in ("k", "v", "k_scale", "v_scale") + (("weights",) if "weights" in s else ()):
        if s[name] is not None:
            x = s[name].view(torch.int8) if s[name].dtype == torch.float8_e4m3fn else s[name]
            x[dst] = x[src]


# ---------------------------------------------------------------------------------------------
# Work and 64-bit values

def _pairs(case):
    """(cached tokens that some row sees, visible (row, token) pairs) over the sequences, for one head.  A tree's rows are
    counted with as many drafted tokens as a chain of half its size has on average."""
    w, sinks = case["window"], case["sinks"]
    tokens = pairs = 0
    for q, kv in zip(*_lengths(case)):
        first = kv - q
        if case["kind"] == "tree":
            seen = min(first, w + sinks) if w else first
            tokens += seen + q
            pairs += q * (seen + max(1, q // 4))
            continue
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
    vector = D * 2 if case["fmt"] == "16" else D + 4
    q_len, kv_len = _lengths(case)
    rows = sum(q_len) * case["q_heads"]
    if case["kind"] == "tree":
        tokens, pairs = _pairs(case)
        mask = sum(q_len) * 4 * -(-max(q_len) // 32)
        return {"bytes": 2 * tokens * H * vector + rows * (4 * D + (4 if case["lse"] else 0)) + mask, "flops": 4 * D * pairs * case["q_heads"]}
    if case["kind"] == "weigh":
        tokens, pairs = _pairs(case)
        held = tokens if case["decay"] == 1.0 else sum(kv_len)
        return {"bytes": H * (tokens * vector + held * (8 if case["decay"] else 4)) + rows * (2 * D + 4), "flops": 2 * D * pairs * case["q_heads"]}
    if case["kind"] == "evict":
        moved = sum(max(0, min(kv, m) - case["sinks"]) for kv, m in zip(kv_len, _budgets(case)) if kv > m)
        lists = 4 * len(kv_len) * case["budget"]
        return {"bytes": H * (4 * sum(kv_len) + lists + moved * (2 * (2 * vector + 4) + 4)), "flops": 0}
    moved = sum(max(0, p - 1) for p in _paths(case))
    return {"bytes": moved * (H * 4 * vector + 4), "flops": 0}


def exact(case, seed):
    if work(case)["flops"] > 8e12:
        return None
    s = _inputs(case, seed)
    q_len, kv_len = s["q_len"], s["kv_len_host"]
    b, H, G, D = case["block"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"]
    w, sinks = case["window"], case["sinks"]

    def cached(name, i, head, kv):
        p = torch.arange(kv, device="cuda")
        blk = s["table"][i].long()[p // b]
        if case["fmt"] == "16":
            return s[name][blk, p % b, head].double()
        return s[name][:, :, head].view(torch.int8)[blk, p % b].view(s[name].dtype).double() * s[name + "_scale"][blk, p % b, head].double()[:, None]

    if case["kind"] in ("evict", "accept"):
        got = {n: s[m].double() for n, m in (("k_cache", "k"), ("v_cache", "v"), ("k_scale", "k_scale"), ("v_scale", "v_scale"), ("weights", "weights"))
               if s.get(m) is not None}
        lists = [[None] * H for _ in kv_len]
        for i, kv in enumerate(kv_len):
            for h in range(H):
                if case["kind"] == "accept":
                    lists[i][h] = (int(s["start"][i]), s["kept"][i, :int(s["count"][i])].long())
                    continue
                p = torch.arange(kv, device="cuda")
                m = min(kv, _budgets(case)[i])
                free = p[sinks:max(sinks, kv - case["recent"])]
                x = s["weights"][s["table"][i].long()[free // b], free % b, h].cpu().numpy()
                best = np.lexsort((np.arange(len(x)), -x))[:max(0, m - min(kv, sinks) - min(max(0, kv - sinks), case["recent"]))]
                keep = np.concatenate([np.arange(min(kv, sinks)), sinks + np.sort(best), np.arange(max(sinks, kv - case["recent"]), kv)])
                lists[i][h] = (0, torch.from_numpy(keep).cuda().long())
        for i in range(len(kv_len)):
            for h in range(H):
                at, src = lists[i][h]
                dst = torch.arange(at, at + len(src), device="cuda")
                t = s["table"][i].long()
                for x in got.values():
                    x[t[dst // b], dst % b, h] = x[t[src // b], src % b, h]
        if case["kind"] == "evict":
            kept = torch.full((len(kv_len), H, case["budget"]), -1, dtype=torch.int32, device="cuda")
            for i in range(len(kv_len)):
                for h in range(H):
                    kept[i, h, :len(lists[i][h][1])] = lists[i][h][1].to(torch.int32)
            got = {"kept": kept, "count": torch.tensor([len(x[0][1]) for x in lists], dtype=torch.int32, device="cuda"), **got}
            order = ("kept", "count", "weights", "k_cache", "v_cache", "k_scale", "v_scale")
            got = {n: got[n] for n in order if n in got}
        return got

    lse_in = prepare(case, seed)["lse"].double() if case["kind"] == "weigh" else None
    out = torch.zeros((s["tokens"], H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], H * G), -math.inf, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if case["kind"] == "weigh" else None
    t0 = 0
    for i, (q, kv) in enumerate(zip(q_len, kv_len)):
        first = kv - q
        j = torch.arange(kv, device="cuda")
        if case["kind"] == "tree":
            bits = s["tree"][t0:t0 + q].cpu().numpy().view(np.uint8)
            path = torch.from_numpy(np.unpackbits(bits, axis=1, bitorder="little")[:, :q]).cuda().bool()
            see = torch.cat([torch.ones((q, first), dtype=torch.bool, device="cuda"), path], 1)
            if w:
                place = see.long().cumsum(1) - 1  # all of the context is on every path
                see &= (place > place[:, -1:] - w) | (place < sinks)
        else:
            at = torch.arange(first, kv, device="cuda")[:, None]
            see = j <= at
            if w:
                see &= (j > at - w) | (j < sinks)
        t, place = s["table"][i].long()[j // b], j % b
        for h in range(H):
            k = cached("k", i, h, kv)
            heads = slice(h * G, (h + 1) * G)
            added = torch.zeros(kv, dtype=torch.float64, device="cuda")
            v = cached("v", i, h, kv) if case["kind"] == "tree" else None
            for r in range(0, q, 1024):
                rows = slice(t0 + r, t0 + min(q, r + 1024))
                x = torch.einsum("tgd,jd->tgj", s["q"][rows, heads].double(), k) / math.sqrt(D)
                x.masked_fill_(~see[r:r + 1024, None, :], -math.inf)
                if case["kind"] == "tree":
                    l = torch.logsumexp(x, -1)
                    out[rows, heads], lse[rows, heads] = torch.exp(x - l[..., None]) @ v, l
                else:
                    added += torch.exp(x - lse_in[rows, heads, None]).sum((0, 1))
            if weights is not None:
                before = case["decay"] * weights[t, place, h] * (j < first) if case["decay"] else 0.0
                weights[t, place, h] = before + added
        t0 += q
    if case["kind"] == "weigh":
        return {"weights": weights}
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
