"""GPU parity of the chunk attention over the paged cache (paged_chunk_fwd)
against its definition in 64 bits, in every element.

Tolerance on O, per element: the weights are rounded to bf16 (half a step, 2^-8
of each), so a weighted sum of values is off by 2^-8 of A = sum_j p_j |v_j|, and
the result's own rounding by 2^-8 of it. The fp32 errors before that (scores,
exponentials, sums of up to 2^13 products) stay below 2^-10 A.
On the LSE: the scores' fp32 sums over d channels, (d + 4) 2^-24 of scale *
sum |q_c k_c|; the row sum's L / 32 + 64 additions, 2^-24 each; its logarithm
and the result's rounding, 2^-21 + 2^-22 |LSE|.
"""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


def _t():
    import torch
    return torch


def _rand(shape, std, seed):
    t = _t()
    g = t.Generator(device="cuda").manual_seed(seed)
    return (t.randn(shape, generator=g, device="cuda") * std).to(t.bfloat16)


def tables(q, kv, P, seed, carts=(), cart_pages=0, spare=2):
    """Page lists: request b starts with the cartridges carts[b], its other pages are private and shuffled."""
    r = np.random.default_rng(seed)
    n_carts = 1 + max([c for cs in carts for c in cs], default=-1)
    need = [-(-L // P) - (len(carts[b]) * cart_pages if carts else 0) for b, L in enumerate(kv)]
    ids = (n_carts * cart_pages + r.permutation(sum(need) + spare)).tolist()
    pages = [[c * cart_pages + j for c in (carts[b] if carts else ()) for j in range(cart_pages)] + [ids.pop() for _ in range(n)]
             for b, n in enumerate(need)]
    return pages, n_carts * cart_pages + sum(need) + spare


def reference(q, kp, vp, counts, kv, pages, scale, g):
    """(O, A, LSE, bound of the scores' error) in 64 bits."""
    t = _t()
    T, Hq, D = sum(counts), q.shape[1], q.shape[2]
    O, A = (t.zeros(T, Hq, D, dtype=t.float64, device="cuda") for _ in range(2))
    LSE, E = (t.zeros(Hq, T, dtype=t.float64, device="cuda") for _ in range(2))
    t0 = 0
    for n, L, pl in zip(counts, kv, pages):
        if n:
            ids = t.tensor(pl, device="cuda")
            K, V = (x[ids].reshape(-1, Hq // g, D)[:L].double() for x in (kp, vp))
            see = t.arange(L, device="cuda")[None, :] <= t.arange(L - n, L, device="cuda")[:, None]
            for h in range(Hq):
                qh, Kh, Vh = q[t0:t0 + n, h].double(), K[:, h // g], V[:, h // g]
                S = (qh @ Kh.T * scale).masked_fill(~see, -np.inf)
                lse = t.logsumexp(S, 1)
                p = (S - lse[:, None]).exp()
                O[t0:t0 + n, h], A[t0:t0 + n, h] = p @ Vh, p @ Vh.abs()
                LSE[h, t0:t0 + n] = lse
                E[h, t0:t0 + n] = ((qh.abs() @ Kh.abs().T) * see).amax(1) * scale * (D + 4) * 2.0 ** -24 + (L / 32 + 64) * 2.0 ** -24
        t0 += n
    return O, A, LSE, E


def compare(o, lse, q, kp, vp, counts, kv, pages, scale, g):
    T = sum(counts)
    O, A, LSE, E = reference(q, kp, vp, counts, kv, pages, scale, g)
    e = (o[:T].double() - O).abs() - (2.0 ** -8 * O.abs() + (2.0 ** -8 + 2.0 ** -10) * A)
    assert not _t().isnan(e).any() and e.max().item() <= 0, (e.max().item(), (e > 0).sum().item(), e.argmax().item())
    e = (lse.double() - LSE).abs() - (E + 2.0 ** -21 + 2.0 ** -22 * LSE.abs())
    assert not _t().isnan(e).any() and e.max().item() <= 0, (e.max().item(), (e > 0).sum().item())


def run(cas, counts, kv, P, Hkv, g, D, seed=1, carts=(), cart_pages=0, scale=None, pad=0, garbage=True, **kw):
    t = _t()
    pages, npages = tables(counts, kv, P, seed, carts, cart_pages)
    scale = scale or float(np.float32(D ** -0.5))
    prob = cas.DecodeProblem(counts, kv, pages, npages, P, Hkv, g, D, scale)
    kp, vp = _rand((npages, P, Hkv, D), 0.7, seed), _rand((npages, P, Hkv, D), 1.0, seed + 1)
    if garbage:   # whatever no request reads: unused pages, and rows behind the last key
        used = t.zeros(npages * P, dtype=t.bool)
        for L, pl in zip(kv, pages):
            for j, p in enumerate(pl):
                used[p * P: p * P + min(P, L - j * P)] = True
        for x in (kp, vp):
            x.view(npages * P, Hkv, D)[~used.cuda()] = float("nan")
    q = _rand((sum(counts) + pad, Hkv * g, D), 1.0, seed + 2)
    o = t.full_like(q, 7.0)
    o2, lse = cas.paged_chunk_fwd(q, kp, vp, prob, o=o, **kw)
    assert o2 is o and (o[sum(counts):] == 7.0).all()
    compare(o, lse, q, kp, vp, counts, kv, pages, scale, g)
    return prob, q, kp, vp, o, lse, pages


@pytest.mark.parametrize("P,D", [(16, 128), (32, 64), (64, 128), (128, 64)])
@pytest.mark.parametrize("Hkv,g", [(1, 1), (2, 4), (3, 3), (8, 8)])
def test_edges(gpu_lib, P, D, Hkv, g):
    """Counts around the 256-row blocks and 64-key tiles, requests without new
    tokens, without keys, and of one token."""
    b = 256 // g
    counts = [1, b - 1, b, 0, b + 1, 5, 1, 2 * b + 3, 0]
    kv = [1, b - 1, b + 64, 9, b + 127, 64, 65, 2 * b + 3 + 1000, 0]
    run(gpu_lib, counts, kv, P, Hkv, g, D, seed=P + D + g, pad=3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [63, 64, 65, 1000, 2047, 8192])
def test_one_short_request(gpu_lib, L, D):
    """The key axis in 1 to many pieces."""
    prob, *_ = run(gpu_lib, [33], [L], 16, 2, 4, D, seed=L)
    info = gpu_lib.chunk_plan(prob)[0]
    assert info.max_partials > 1 or L < 8192


def test_single_tokens(gpu_lib):
    run(gpu_lib, [1] * 20, [1 + 97 * i for i in range(20)], 16, 4, 4, 128)
    run(gpu_lib, [1], [5000], 16, 8, 5, 128)


@pytest.mark.parametrize("D,Hkv,g", [(128, 4, 4), (64, 8, 3)])
def test_single_tokens_over_shared_cartridges(gpu_lib, D, Hkv, g):
    """Runs of decode requests that read the same cartridges, before, between and
    behind chunks: through the decode kernels, with and without LSE, captured, and
    with a workspace that holds something else before."""
    t = _t()
    share = [[0, 1, 2, 3], [2, 0, 3, 1], [3], [1, 2]] * 4
    carts = share + [[0, 1]] + share[:9] + [[], [2]] + share[3:] + [[]]
    counts = [1] * 16 + [150] + [1] * 8 + [0] + [40, 300] + [1] * 13 + [2]
    kv = [512 * len(c) + 9 + 5 * i + n for i, (c, n) in enumerate(zip(carts, counts))]
    prob, q, kp, vp, o, lse, pages = run(gpu_lib, counts, kv, 16, Hkv, g, D, carts=carts, cart_pages=32, pad=2)
    info = gpu_lib.chunk_plan(prob)[0]
    assert info.decode_parts == 0 or info.decode_tokens >= 8
    many = [1] * 40
    mkv = [512 * 4 * 4 + 1 + 3 * i for i in range(40)]
    prob, q, kp, vp, o, lse, pages = run(gpu_lib, many, mkv, 16, Hkv, g, D, seed=9, carts=[list(range(16))] * 40, cart_pages=32, pad=1)
    info = gpu_lib.chunk_plan(prob)[0]
    assert (info.decode_parts, info.decode_tokens, info.workgroups) == (1, 40, 0)
    ws = t.full((info.ws_bytes,), 255, dtype=t.uint8, device="cuda")
    a, none = gpu_lib.paged_chunk_fwd(q, kp, vp, prob, need_lse=False, workspace=ws)
    assert none is None and t.equal(a[:40], o[:40])
    mixed, mk = [1] * 20 + [70] + [1] * 20, mkv[:20] + [512 * 16 + 70] + mkv[20:]
    prob, q, kp, vp, o, lse, pages = run(gpu_lib, mixed, mk, 16, Hkv, g, D, seed=11, carts=[list(range(16))] * 41, cart_pages=32)
    info = gpu_lib.chunk_plan(prob)[0]
    assert (info.decode_parts, info.decode_tokens) == (2, 40) and info.workgroups > 0
    o2, lse2 = t.zeros_like(o), t.zeros_like(lse)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        gpu_lib.paged_chunk_fwd(q, kp, vp, prob, o=o2, lse=lse2)
    for i in range(3):
        q.copy_(_rand(q.shape, 1.0, 70 + i))
        graph.replay()
        want = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
        t.cuda.synchronize()
        assert t.equal(o2, want[0]) and t.equal(lse2, want[1])


def test_shared_cartridges_and_a_long_chunk(gpu_lib):
    run(gpu_lib, [700, 1, 33, 300], [700 + 1024 + 60, 512 + 5, 1024 + 512 + 33, 300], 32, 2, 4, 128, seed=3,
        carts=[[2, 0], [1], [0, 1, 2], []], cart_pages=16)
    run(gpu_lib, [1100], [4000], 64, 1, 12, 64, seed=4)


@pytest.mark.parametrize("D", [64, 128])
def test_rising_scores(gpu_lib, D):
    """Keys whose scores lie 40 and 150 above everything before them: a running
    maximum moves, a fixed reference overflows."""
    t = _t()
    counts, kv = [130], [130 + 700]
    pages, npages = tables(counts, kv, 16, 5)
    prob = gpu_lib.DecodeProblem(counts, kv, pages, npages, 16, 1, 2, D, 1.0)
    q = t.full((130, 2, D), 0.25, dtype=t.bfloat16, device="cuda")
    kp, vp = _rand((npages, 16, 1, D), 0.05, 6), _rand((npages, 16, 1, D), 1.0, 7)
    for key, score in ((300, 40.0), (600, 150.0), (760, 170.0)):
        kp[pages[0][key // 16], key % 16] = score * 4 / D
    o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    compare(o, lse, q, kp, vp, counts, kv, pages, 1.0, 2)


@pytest.mark.parametrize("D", [64, 128])
def test_values_past_a_query_do_not_reach_it(gpu_lib, D):
    """NaN and infinities in the keys and values of new tokens 70 and 90 of 150:
    the queries before them are what they were, the ones after get them."""
    t = _t()
    counts, kv, P, Hkv, g = [150, 3], [150 + 300, 40], 16, 2, 2
    pages, npages = tables(counts, kv, P, 8)
    prob = gpu_lib.DecodeProblem(counts, kv, pages, npages, P, Hkv, g, D, 0.1)
    q, kp, vp = _rand((153, 4, D), 1.0, 1), _rand((npages, P, Hkv, D), 0.7, 2), _rand((npages, P, Hkv, D), 1.0, 3)
    o0, l0 = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    at = lambda i: (pages[0][(300 + i) // P], (300 + i) % P)
    v2 = vp.clone()
    v2[at(70)][0, 3] = float("inf")
    v2[at(70)][0, D - 1] = float("-inf")
    v2[at(90)][1, 5] = float("nan")
    o, lse = gpu_lib.paged_chunk_fwd(q, kp, v2, prob)
    assert (o[70:150, :2, 3] == float("inf")).all() and (o[70:150, :2, D - 1] == float("-inf")).all()
    assert t.isnan(o[90:150, 2:, 5]).all()
    want, got = o0.clone(), o.clone()
    for x in (want, got):
        x[70:150, :2, [3, D - 1]] = 0
        x[90:150, 2:, 5] = 0
    # (the pass that keeps them apart may round in another order)
    _, A, LSE, E = reference(q, kp, vp, counts, kv, pages, 0.1, g)
    assert ((want.double() - got.double()).abs() <= 2.0 ** -6 * A + 2.0 ** -7 * want.double().abs()).all()
    assert ((lse.double() - LSE).abs() <= E + 2.0 ** -21 + 2.0 ** -22 * LSE.abs()).all()
    k2 = kp.clone()
    k2[at(70)][0] = float("nan")
    o, lse = gpu_lib.paged_chunk_fwd(q, k2, vp, prob)
    assert t.isnan(o[70:150, :2]).all() and t.isnan(lse[:2, 70:150]).all()
    assert t.isfinite(o[:70]).all() and t.isfinite(o[150:]).all() and t.isfinite(o[:, 2:]).all() and t.isfinite(lse[:, :70]).all()
    k2[at(70)][0] = float("inf")
    o, lse = gpu_lib.paged_chunk_fwd(q, k2, vp, prob)
    assert t.isfinite(o[:70]).all() and t.isfinite(o[:, 2:]).all() and t.isfinite(lse[:, :70]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,Hkv,g", [(16, 2, 1), (32, 1, 4), (128, 3, 5)])
def test_few_rows(gpu_lib, P, Hkv, g, D):
    """Blocks of 1 to 65 rows, which divide the keys among the waves up to 64:
    fewer keys than waves, ends inside a tile's halves, pieces of long ones."""
    for rows in (1, 31, 32, 33, 63, 64, 65):
        n = max(1, rows // g)
        counts = [n, 1, n, n, n + 1, n]
        kv = [n, 33, n + 31, n + 64, n + 257, 6000]
        run(gpu_lib, counts, kv, P, Hkv, g, D, seed=rows)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [12, 28])
def test_few_rows_rising_and_not_finite(gpu_lib, n, D):
    """24 and 56 rows: scores 40 to 170 above those before them, in keys of every
    wave; NaN and infinities in keys and values of a new token reach the queries
    from it on and no other."""
    t = _t()
    L = 700 + n
    pages, npages = tables([n], [L], 16, 5)
    at = lambda key: (pages[0][key // 16], key % 16)
    prob = gpu_lib.DecodeProblem([n], [L], pages, npages, 16, 1, 2, D, 1.0)
    q = t.full((n, 2, D), 0.25, dtype=t.bfloat16, device="cuda")
    kp, vp = _rand((npages, 16, 1, D), 0.05, 6), _rand((npages, 16, 1, D), 1.0, 7)
    for key, score in ((100, 40.0), (350, 150.0), (600, 160.0), (705, 170.0)):
        kp[at(key)] = score * 4 / D
    o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    compare(o, lse, q, kp, vp, [n], [L], pages, 1.0, 2)
    kp = _rand((npages, 16, 1, D), 0.7, 6)
    q = _rand((n, 2, D), 1.0, 8)
    prob = gpu_lib.DecodeProblem([n], [L], pages, npages, 16, 1, 2, D, 0.1)
    bad = 7
    before = [bad], [700 + bad]   # the queries ahead of it, as a request of their own
    for value in ("nan", "inf", "-inf"):
        v2, k2 = vp.clone(), kp.clone()
        v2[at(700 + bad)][0, 3] = float(value)
        k2[at(700 + bad)][0, 2] = float(value)
        o, lse = gpu_lib.paged_chunk_fwd(q, kp, v2, prob)
        compare(o[:bad], lse[:, :bad], q[:bad], kp, vp, *before, pages, 0.1, 2)
        assert (t.isnan(o[bad:, :, 3]) if value == "nan" else o[bad:, :, 3] == float(value)).all()
        assert t.isfinite(o[:, :, [c for c in range(D) if c != 3]]).all()
        o, lse = gpu_lib.paged_chunk_fwd(q, k2, vp, prob)
        compare(o[:bad], lse[:, :bad], q[:bad], kp, vp, *before, pages, 0.1, 2)
        if value == "nan":
            assert t.isnan(o[bad:]).all() and t.isnan(lse[:, bad:]).all()


def test_agrees_with_decode_and_repeats(gpu_lib):
    """The same problem through paged_decode_fwd (both within half a step of the
    weights and of the result), and the same bits on a second call."""
    prob, q, kp, vp, o, lse, pages = run(gpu_lib, [3, 1, 60], [900, 77, 1500], 16, 2, 4, 128, garbage=False)
    t = _t()
    o2, lse2 = gpu_lib.paged_decode_fwd(q, kp, vp, [3, 1, 60], [900, 77, 1500], pages, 2, 4, 128 ** -0.5)
    _, A, _, E = reference(q, kp, vp, [3, 1, 60], [900, 77, 1500], pages, 128 ** -0.5, 4)
    assert ((o.double() - o2.double()).abs() <= 2.0 ** -7 * o2.double().abs() + 2.0 ** -6 * A).all()
    assert ((lse - lse2).double().abs() <= 2 * (E + 2.0 ** -20 + 2.0 ** -21 * lse.abs())).all()
    o3, lse3 = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    assert t.equal(o, o3) and t.equal(lse, lse3)


def test_no_lse_and_workspaces(gpu_lib):
    t = _t()
    prob, q, kp, vp, o, lse, _ = run(gpu_lib, [40], [3000], 16, 2, 4, 128)
    n = gpu_lib.paged_chunk_workspace_size(prob)
    ws = t.full((n + 256,), 255, dtype=t.uint8, device="cuda")
    a, none = gpu_lib.paged_chunk_fwd(q, kp, vp, prob, need_lse=False, workspace=ws[:n])
    assert none is None and t.equal(a, o) and (ws[n:] == 255).all()
    b, _ = gpu_lib.paged_chunk_fwd(q, kp, vp, prob, workspace=ws[:1])      # too small: one of its own
    assert t.equal(b, o)


def test_streams(gpu_lib):
    t = _t()
    prob, q, kp, vp, o, lse, _ = run(gpu_lib, [300, 1], [2000, 900], 16, 2, 4, 128)
    ss = [t.cuda.Stream() for _ in range(2)]
    t.cuda.synchronize()
    outs = [gpu_lib.paged_chunk_fwd(q, kp, vp, prob, stream=ss[i % 2]) for i in range(6)]   # two calls at once
    t.cuda.synchronize()
    for a, b in outs:
        assert t.equal(a, o) and t.equal(b, lse)


def test_graphs(gpu_lib):
    """Captured calls, replayed with other inputs and eager calls between them;
    two graphs with a workspace each."""
    t = _t()
    cases = [run(gpu_lib, c, kv, 16, 2, 4, 128, seed=s) for c, kv, s in (([40, 1], [3000, 50], 1), ([300], [700], 2))]
    graphs = []
    for prob, q, kp, vp, o, lse, _ in cases:
        ws = t.empty(gpu_lib.paged_chunk_workspace_size(prob), dtype=t.uint8, device="cuda")
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            gpu_lib.paged_chunk_fwd(q, kp, vp, prob, o=o, lse=lse, workspace=ws)
        graphs.append((g, ws))
    for i in range(3):
        for (prob, q, kp, vp, o, lse, _), (g, ws) in zip(cases, graphs):
            q.copy_(_rand(q.shape, 1.0, 100 + i))
            o.zero_()
            lse.zero_()
            g.replay()
        for prob, q, kp, vp, o, lse, _ in cases:
            o2, lse2 = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
            t.cuda.synchronize()
            assert t.equal(o, o2) and t.equal(lse, lse2)


@pytest.mark.parametrize("D,Hkv,g", [(128, 8, 4), (64, 3, 5)])
def test_calls_without_tables(gpu_lib, D, Hkv, g):
    """Few whole blocks, whose tables are kernel arguments: an empty workspace, calls
    on two streams at once, and a captured call replayed with other inputs."""
    t = _t()
    counts, kv = [0, 33, 1, 0, 20, 5], [9, 500, 260, 0, 20, 70]
    prob, q, kp, vp, o, lse, _ = run(gpu_lib, counts, kv, 16, Hkv, g, D, pad=2)
    assert gpu_lib.paged_chunk_workspace_size(prob) == 0
    a, b = gpu_lib.paged_chunk_fwd(q, kp, vp, prob, workspace=t.empty(0, dtype=t.uint8, device="cuda"))
    ss = [t.cuda.Stream() for _ in range(2)]
    t.cuda.synchronize()
    outs = [gpu_lib.paged_chunk_fwd(q, kp, vp, prob, stream=ss[i % 2]) for i in range(6)] + [(a, b)]
    t.cuda.synchronize()
    n = sum(counts)
    assert all(t.equal(x[:n], o[:n]) and t.equal(y, lse) for x, y in outs)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        gpu_lib.paged_chunk_fwd(q, kp, vp, prob, o=o, lse=lse)
    for i in range(3):
        q.copy_(_rand(q.shape, 1.0, 30 + i))
        lse.zero_()
        graph.replay()
        x, y = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
        t.cuda.synchronize()
        assert t.equal(x[:n], o[:n]) and t.equal(y, lse)


def test_pages_past_4_gib(gpu_lib):
    t = _t()
    P, Hkv, D, n = 128, 64, 128, 2600
    kp, vp = (t.zeros((n, P, Hkv, D), dtype=t.bfloat16, device="cuda") for _ in range(2))
    pages = [[n - 1, 3, n - 2]]
    for p in pages[0]:
        kp[p], vp[p] = _rand((P, Hkv, D), 0.7, p), _rand((P, Hkv, D), 1.0, p + 1)
    prob = gpu_lib.DecodeProblem([140], [300], pages, n, P, Hkv, 1, D, 0.09)
    q = _rand((140, Hkv, D), 1.0, 5)
    o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    compare(o, lse, q, kp, vp, [140], [300], pages, 0.09, 1)


@pytest.mark.parametrize("seed", range(24))
def test_random_problems(gpu_lib, seed):
    """Seeded problems: head layouts, page sizes, cartridges in common, ragged
    chunks, single tokens and empty requests in any order."""
    r = np.random.default_rng(5000 + seed)
    P, D = int(r.choice([16, 32, 64, 128])), int(r.choice([64, 128]))
    Hkv, g, B = int(r.choice([1, 2, 3, 4, 6, 8])), int(r.choice([1, 2, 3, 4, 5, 7, 8])), int(r.integers(1, 14))
    cart_pages = int(r.integers(1, 700 // P + 2))
    carts, counts, kv = [], [], []
    for _ in range(B):
        c = r.permutation(5)[: int(r.integers(0, 5))].tolist()
        n = int(r.choice([0, 1, 1, 1, int(r.integers(2, 40)), int(r.integers(40, 500))]))
        own = n + int(r.choice([0, int(r.integers(0, 70)), int(r.integers(0, 900))]))
        carts.append(c)
        counts.append(n)
        kv.append(len(c) * cart_pages * P + own)
    if not sum(counts):
        counts[0], kv[0] = 1, kv[0] + 1
    run(gpu_lib, counts, kv, P, Hkv, g, D, seed=seed, carts=carts, cart_pages=cart_pages, pad=int(r.integers(0, 3)))


def test_host_threads(gpu_lib):
    """Four threads with a stream each: attention on one shared problem, and
    appending to pools of their own."""
    import threading
    t = _t()
    prob, q, kp, vp, o, lse, pages = run(gpu_lib, [300, 1, 40], [2000, 900, 777], 16, 2, 4, 128)
    rope = gpu_lib.Rope(128, 1e4)
    aprob = gpu_lib.DecodeProblem([3, 1], [20, 33], [[0, 1], [2, 3, 4]], 5, 16, 2, 4, 128, 0.1)
    x = _rand((4, 2, 128), 1.0, 5)
    pools = [[t.zeros((5, 16, 2, 128), dtype=t.bfloat16, device="cuda") for _ in range(2)] for _ in range(5)]
    gpu_lib.paged_append(x, x, *pools[4], aprob, rope=rope)
    t.cuda.synchronize()
    bad = []

    def work(i):
        try:
            s = t.cuda.Stream()
            for _ in range(20):
                a, b = gpu_lib.paged_chunk_fwd(q, kp, vp, prob, stream=s)
                gpu_lib.paged_append(x, x, *pools[i], aprob, rope=rope, stream=s)
                s.synchronize()
                if not (t.equal(a, o) and t.equal(b, lse) and t.equal(pools[i][0], pools[4][0])):
                    bad.append(i)
        except Exception as e:   # noqa: BLE001
            bad.append(e)
    ths = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for th in ths:
        th.start()
    for th in ths:
        th.join()
    assert not bad


def test_serving_steps(gpu_lib):
    """Prompts prefilled in two chunks, then decoded token by token, positions and
    cache through paged_append: every step's attention against the whole
    sequence's, whose keys are rotated in 64 bits and rounded once. (A rotated
    value next to a rounding border may fall to the other side, one step of 2^-7:
    a query or key channel off by that moves a score by scale * 2^-7 |q_c k_c|,
    and no pair of channels does so in more than a fraction of the rows, so the
    weights' bound is taken four times.)"""
    t = _t()
    Hkv, g, D, P, cart = 2, 2, 64, 16, 64
    Hq, scale = Hkv * g, 0.125
    rope = gpu_lib.Rope(D, 1e4)
    lens = [150, 37]                                   # prompt and generated tokens
    steps = [[100, 20], [48, 15], [1, 1], [1, 1]]
    own = [[4 + 2 * j for j in range(10)], [5 + 2 * j for j in range(10)]]
    npages = 4 + 20
    kp, vp = (t.zeros((npages, P, Hkv, D), dtype=t.bfloat16, device="cuda") for _ in range(2))
    ck, cv = _rand((cart, Hkv, D), 0.7, 1), _rand((cart, Hkv, D), 1.0, 2)
    kp[:4], vp[:4] = ck.view(4, P, Hkv, D), cv.view(4, P, Hkv, D)
    X = [_rand((n, Hq + 2 * Hkv, D), 1.0, 3 + i) for i, n in enumerate(lens)]
    done = [0, 0]
    full = []
    for i in range(2):
        pos = np.arange(lens[i]) + cart
        rot = lambda x: t.from_numpy(oracle.rope.rotate(x.double().cpu().numpy(), pos, rope.turns)).cuda().to(t.bfloat16)
        full.append((rot(X[i][:, :Hq]), t.cat([ck, rot(X[i][:, Hq:Hq + Hkv])]), t.cat([cv, X[i][:, Hq + Hkv:]])))
    for counts in steps:
        kv = [cart + d + n for d, n in zip(done, counts)]
        pages = [([0, 1, 2, 3] + o)[: -(-L // P)] for o, L in zip(own, kv)]
        prob = gpu_lib.DecodeProblem(counts, kv, pages, npages, P, Hkv, g, D, scale)
        x = t.cat([X[i][done[i]: done[i] + counts[i]] for i in range(2)])
        q = gpu_lib.paged_append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], kp, vp, prob, rope=rope, q=x[:, :Hq])
        o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
        if counts == [1, 1]:
            o, lse = gpu_lib.paged_decode_fwd(q, kp, vp, counts, kv, pages, Hkv, g, scale, problem=prob)
        t0 = 0
        for i, n in enumerate(counts):
            Q, K, V = full[i]
            L = kv[i]
            one, flat = [list(range(L))], lambda y: y[:L].reshape(L, 1, Hkv, D)
            O, A, LSE, E = reference(Q[done[i]: done[i] + n], flat(K), flat(V), [n], [L], one, scale, g)
            assert ((o[t0:t0 + n].double() - O).abs() <= 2.0 ** -8 * O.abs() + 4 * 2.0 ** -8 * A).all()
            assert ((lse[:, t0:t0 + n].double() - LSE).abs() <= 4 * 2.0 ** -8).all()
            t0 += n
        done = [d + n for d, n in zip(done, counts)]
    assert done == lens
