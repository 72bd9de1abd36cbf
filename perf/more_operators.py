"""Performance cases of the operators around a cache that beams share: choosing the beams, moving their states, moving pages.

* ``select``   beam_select: the best continuations over all beams and the vocabulary of every batch entry, from the logits
               of the beams' last tokens. Returns their scores, parents (beams) and tokens.
* ``reorder``  beam_reorder: states kept per beam (token histories, dense caches) follow the surviving beams' parents.
               Returns the new states.
* ``pages``    pages_copy: whole pages or the first rows of some go to other pages, in the page pools of every layer: the
               tails of forked sequences, and the moves that make a cache compact. Returns the pools.

The sizes of a case are plain values; what they leave open (parents, which pages move, which beams have ended) comes from
``shape_seed``, what the tensors hold from the seed.
"""
import math
import random

import numpy as np
import torch

DEV = "cuda"
own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "int32": torch.int32, "uint8": torch.uint8}
_BYTES = {"bf16": 2, "fp32": 4, "int32": 4, "uint8": 1}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _named(c, name):
    return dict(name=name, **c) if name else c


def _select(name=None, **kw):
    # pad: further columns of the logits' rows that are no tokens (a projection padded to its tiles). ended: share of the
    # beams that are finished; banned: share of each row's tokens at -inf; empty: a beam whose tokens are all at -inf.
    c = dict(kind="select", dtype="bf16", batch=1, beams=4, vocab=32000, pad=0, k=8, ended=0.0, banned=0.0, empty=0, shape_seed=1)
    c.update(kw)
    return _named(c, name)


def _reorder(name=None, **kw):
    # tensors: states moved in one call, each [batch, beams, capacity, width] of which the first `used` of the capacity count.
    c = dict(kind="reorder", dtype="int32", tensors=1, batch=1, beams=4, capacity=256, used=100, width=1, shape_seed=1)
    c.update(kw)
    return _named(c, name)


def _pages(name=None, **kw):
    # pools: K and V of every layer. whole: whole pages move (compaction); otherwise their first 1 to page rows do, and a
    # page may be copied more than once (the children of one beam).
    c = dict(kind="pages", dtype="bf16", pools=2, page=16, kv_heads=8, head_dim=128, copies=8, whole=0, spare=64, shape_seed=1)
    c.update(kw)
    return _named(c, name)


def listed():
    return [
        # One request with four beams, each step of its decoding: latency.
        _select("select_1x4_32k"),
        # A serving batch's step: 16 requests of 8 beams, a vocabulary of odd size, a few beams have ended.
        _select("select_16x8_130k", batch=16, beams=8, vocab=130001, k=16, ended=0.1),
        # The largest batch: 64 requests of 8 beams.
        _select("select_64x8_131k", batch=64, beams=8, vocab=131072, k=16),
        # fp32 logits, in which a model is checked, constrained to some of the tokens, in padded rows; one beam has none left.
        _select("select_fp32_odd", dtype="fp32", batch=6, beams=5, vocab=49999, pad=17, k=10, ended=0.1, banned=0.6, empty=1),
        # The token histories of one request's beams: latency.
        _reorder("reorder_history", batch=1, beams=4, capacity=512, used=211),
        # A serving batch's histories of odd lengths: tokens, their log-probabilities, and two more of the kind.
        _reorder("reorder_4_histories", tensors=4, batch=64, beams=8, capacity=2048, used=777),
        # The beams' own keys and values in a dense cache: 200 of 256 tokens of 8 heads of 128.
        _reorder("reorder_dense_cache", dtype="bf16", tensors=2, batch=32, beams=8, capacity=256, used=200, width=1024),
        # One request's beams fork, in one layer: latency.
        _pages("fork_4_1layer", copies=4),
        # A serving batch's beams fork: the tails of 200 of them in the 64 pools of 32 layers.
        _pages("fork_200_32layers", pools=64, copies=200, spare=200),
        # A layer's cache is made compact: 8,192 whole pages move.
        _pages("compact_8k", copies=8192, whole=1, spare=300),
        # A small model in fp32: three heads of 64, wider pages, odd counts.
        _pages("fork_odd_fp32", dtype="fp32", pools=10, page=64, kv_heads=3, head_dim=64, copies=37, spare=11),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["select", "select", "reorder", "pages"])
    seed = rng.randrange(1, 1 << 20)
    while True:
        if kind == "select":
            beams = rng.choice([1, 2, 3, 4, 5, 8, 8, 12, 16, 32])
            c = _select(dtype=rng.choice(["bf16", "bf16", "fp32"]), batch=_logint(rng, 1, 64), beams=beams,
                        vocab=_logint(rng, 1000, 131072), pad=rng.choice([0, 0, rng.randint(1, 64)]),
                        k=rng.randint(beams, min(64, 2 * beams)), ended=rng.choice([0.0, 0.0, 0.2]),
                        banned=rng.choice([0.0, 0.0, 0.5, 0.99]), empty=rng.choice([0, 0, 1]), shape_seed=seed)
        elif kind == "reorder":
            dense, capacity = rng.random() < 0.5, _logint(rng, 8, 2048)
            c = _reorder(dtype=rng.choice(["bf16", "fp32"] if dense else ["int32", "fp32", "uint8", "bf16"]),
                         tensors=rng.randint(1, 8), batch=_logint(rng, 1, 64), beams=rng.randint(2, 16), capacity=capacity,
                         used=_logint(rng, 1, capacity), width=_logint(rng, 16, 1024) if dense else rng.choice([1, 1, 3]),
                         shape_seed=seed)
        else:
            c = _pages(dtype=rng.choice(["bf16", "bf16", "fp32", "uint8"]), pools=2 * _logint(rng, 1, 32),
                       page=rng.choice([16, 16, 32, 64, 128]), kv_heads=rng.choice([1, 2, 3, 4, 8]), head_dim=rng.choice([64, 128]),
                       copies=_logint(rng, 1, 8192), whole=int(rng.random() < 0.4), spare=_logint(rng, 1, 300), shape_seed=seed)
        most = {"select": 1.34e8, "reorder": 3e8, "pages": 1.07e9}[kind]
        if work(c)["bytes"] <= most and _held(c) <= 4e9:
            return c


# ---------------------------------------------------------------------------
# Shapes (from the case alone)
# ---------------------------------------------------------------------------
def _beam_flags(c):
    """Which beams have ended, and which one has no token left (or -1), of every batch entry."""
    r = random.Random(c["shape_seed"])
    ended = [[r.random() < c["ended"] for _ in range(c["beams"])] for _ in range(c["batch"])]
    return ended, [r.randrange(c["beams"]) if c["empty"] else -1 for _ in range(c["batch"])]


def _parents(c):
    """Few beams of a request survive a step, and those have several children."""
    r = random.Random(c["shape_seed"])
    return [sorted(int(c["beams"] * r.random() ** 2) for _ in range(c["beams"])) for _ in range(c["batch"])]


def _page_copies(c):
    """(copies [n, 3] of source page, page and rows, pages of the pool)."""
    r = random.Random(c["shape_seed"])
    n, P = c["copies"], c["page"]
    pages = 2 * n + c["spare"]
    if c["whole"]:
        # The used pages behind the first n + spare go to free ones ahead of them.
        ids = list(range(pages - n, pages))
        free = sorted(r.sample(range(pages - n), n))
        return np.array([[s, d, P] for s, d in zip(reversed(ids), free)], dtype=np.int32), pages
    ids = r.sample(range(pages), 2 * n)
    return np.array([[ids[int(n * r.random())], ids[n + i], r.randint(1, P)] for i in range(n)], dtype=np.int32), pages


def _held(c):
    """Bytes of the tensors that a case's state has."""
    size = _BYTES[c["dtype"]]
    if c["kind"] == "select":
        return c["batch"] * c["beams"] * (c["vocab"] + c["pad"]) * size
    if c["kind"] == "reorder":
        return 2 * c["tensors"] * c["batch"] * c["beams"] * c["capacity"] * c["width"] * size
    return c["pools"] * (2 * c["copies"] + c["spare"]) * c["page"] * c["kv_heads"] * c["head_dim"] * size


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _values(gen, shape, dtype):
    if dtype in ("int32", "uint8"):
        return torch.randint(0, 1 << 30 if dtype == "int32" else 256, shape, generator=gen, device=DEV, dtype=_TYPES[dtype])
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(_TYPES[dtype])


def _inputs(c, seed):
    gen = _gen(seed)
    if c["kind"] == "select":
        B, N, V = c["batch"], c["beams"], c["vocab"]
        # Most tokens are noise; one in a thousand stands out, as a language model's logits have it.
        x = torch.randn((B, N, V + c["pad"]), generator=gen, device=DEV)
        x = 2.0 * x + 4.0 * (torch.rand(x.shape, generator=gen, device=DEV) < 1e-3)
        if c["banned"]:
            x.masked_fill_(torch.rand(x.shape, generator=gen, device=DEV) < c["banned"], -math.inf)
        ended, empty = _beam_flags(c)
        for b, i in enumerate(empty):
            if i >= 0:
                x[b, i] = -math.inf
        x[..., V:] = 1e4
        scores = -5.0 - 3.0 * torch.rand((B, N), generator=gen, device=DEV)
        return dict(logits=x.to(_TYPES[c["dtype"]])[..., :V], scores=scores, finished=torch.tensor(ended, device=DEV))
    if c["kind"] == "reorder":
        shape = (c["batch"], c["beams"], c["capacity"], c["width"])
        xs = [_values(gen, shape, c["dtype"]) for _ in range(c["tensors"])]
        return dict(xs=[x[:, :, :c["used"]] for x in xs], parents=torch.tensor(_parents(c), dtype=torch.int32, device=DEV))
    copies, pages = _page_copies(c)
    pools = _values(gen, (c["pools"], pages, c["page"], c["kv_heads"], c["head_dim"]), c["dtype"])
    return dict(copies=copies, pools=pools)


def prepare(case, seed):
    s = dict(c=case, **_inputs(case, seed))
    if case["kind"] == "reorder":
        # A program with states per beam has two sets of them, and goes from one to the other.
        s["outs"] = [torch.zeros((c0, c1, case["capacity"], c3), dtype=x.dtype, device=DEV)[:, :, :c2]
                     for x in s["xs"] for c0, c1, c2, c3 in [x.shape]]
    if own and case["kind"] == "pages":
        import paper_2606_04557_amd as cas
        s["cache"] = cas.PagePools(list(s["pools"].unbind(0)))
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2606_04557_amd as cas
    c = s["c"]
    if c["kind"] == "select":
        scores, parents, tokens = cas.beam_select(s["logits"], s["scores"], c["k"], finished=s["finished"], pad_token=0)
        return {"scores": scores, "parents": parents, "tokens": tokens}
    if c["kind"] == "reorder":
        return {"ys": cas.beam_reorder(s["xs"], s["parents"], outs=s["outs"])}
    cas.pages_copy(s["cache"], s["copies"])
    return {"pools": s["pools"]}


# ---------------------------------------------------------------------------
# The plain form: elementary operations; scores in 64 bits, which two beams' candidates may need to be told apart
# ---------------------------------------------------------------------------
def _run_plain(s):
    c = s["c"]
    if c["kind"] == "select":
        return _plain_select(s["logits"], s["scores"], s["finished"], c["k"])
    if c["kind"] == "reorder":
        batch = torch.arange(c["batch"], device=DEV)[:, None]
        for x, y in zip(s["xs"], s["outs"]):
            y.copy_(x[batch, s["parents"].long()])
        return {"ys": s["outs"]}
    src, dst, rows = s["copies"].astype(np.int64).T
    row = np.arange(rows.sum()) - np.repeat(np.cumsum(rows) - rows, rows)
    at = [torch.from_numpy(np.repeat(p, rows) * c["page"] + row).to(DEV) for p in (src, dst)]
    flat = s["pools"].view(c["pools"], -1, c["kv_heads"] * c["head_dim"])
    flat[:, at[1]] = flat[:, at[0]]
    return {"pools": s["pools"]}


def _plain_select(logits, scores, finished, k):
    B, N, V = logits.shape
    x = logits.double()
    m = x.amax(-1, keepdim=True)
    x = x - m
    x = x - x.exp().sum(-1, keepdim=True).log()
    x = x + scores.double()[..., None]
    # (The row of a beam without a token is -inf - -inf = NaN here.)
    x = torch.where(x.isnan() | finished[..., None], -math.inf, x)
    x[..., 0] = torch.where(finished, scores.double(), x[..., 0])
    # (A stable sort: of equal candidates the first stays first.)
    best, at = torch.sort(x.view(B, N * V), dim=1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k]
    return {"scores": best.float(), "parents": (at // V).int(), "tokens": (at % V).int()}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "select":
        live = sum(not e for row in _beam_flags(c)[0] for e in row)
        return {"bytes": live * c["vocab"] * _BYTES[c["dtype"]] + 5 * c["batch"] * c["beams"] + 12 * c["batch"] * c["k"],
                "flops": 4 * live * c["vocab"]}
    if c["kind"] == "reorder":
        row = c["tensors"] * c["used"] * c["width"] * _BYTES[c["dtype"]]
        return {"bytes": sum((len(set(p)) + len(p)) * row + 4 * len(p) for p in _parents(c)), "flops": 0}
    copies, _ = _page_copies(c)
    read = {}   # a page that several children copy is read once
    for s, _, n in copies.tolist():
        read[s] = max(read.get(s, 0), n)
    row = c["pools"] * c["kv_heads"] * c["head_dim"] * _BYTES[c["dtype"]]
    return {"bytes": (sum(read.values()) + int(copies[:, 2].sum())) * row, "flops": 0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = case
    t = _inputs(c, seed)
    if c["kind"] == "reorder":   # (moves of values, one by one)
        return {"ys": [torch.stack([torch.stack([x[b, p] for p in row]) for b, row in enumerate(_parents(c))]) for x in t["xs"]]}
    if c["kind"] == "pages":
        pools = t["pools"].clone()
        for s, d, n in t["copies"].tolist():
            pools[:, d, :n] = t["pools"][:, s, :n]
        return {"pools": pools}
    k, V = c["k"], c["vocab"]
    out = {"scores": [], "parents": [], "tokens": []}
    for x, score, ended in zip(t["logits"], t["scores"].double(), t["finished"]):
        # One batch entry: every beam's candidates by themselves, then the best of all of them in a list's order.
        found = []
        for i in range(c["beams"]):
            z = x[i].to(torch.float64)
            total = torch.logsumexp(z, 0)
            if ended[i]:
                found.append((-float(score[i]), i, 0))
            elif bool(torch.isfinite(total)):
                least = torch.topk(z, min(k, V)).values[-1]
                at = torch.nonzero((z >= least) & (z > -math.inf))[:, 0]
                found += [(-v, i, j) for v, j in zip((score[i] + (z[at] - total)).tolist(), at.tolist())]
        found = sorted(found)[:k]
        if len(found) < k:   # the first ones of those that are not possible
            have = {(i, j) for _, i, j in found}
            rest = ((math.inf, n // V, n % V) for n in range(2 * k) if (n // V, n % V) not in have)
            found += [f for f, _ in zip(rest, range(k - len(found)))]
        for name, values in zip(("scores", "parents", "tokens"), zip(*found)):
            out[name].append(values)
    return {"scores": -torch.tensor(out["scores"], dtype=torch.float64, device=DEV),
            "parents": torch.tensor(out["parents"], dtype=torch.int32, device=DEV),
            "tokens": torch.tensor(out["tokens"], dtype=torch.int32, device=DEV)}
