"""A whole beam search over the paged cache on the GPU: selection, forked pages,
appending and attention together, as a decoding loop has them.

The model is one attention layer whose queries, keys and values are tables by
token and whose logits are a projection of its output. After every step the
selection is the oracle's for the logits that it saw, the pages of every beam
hold the keys and values of its own tokens in every bit, and the attention is the
oracle's over them (bf16 output: 2e-2 of the largest value, as in the other parity tests)."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

Hkv, G, D, V, PAGE = 2, 2, 64, 301, 16


def _run(cas, beams, prompts, steps, end_token, bias, decode, seed, shared=48, num_pages=400):
    import torch
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)
    kt, vt, qt = rand(V, Hkv, D), rand(V, Hkv, D), rand(V, Hkv * G, D)
    wu = (torch.randn((Hkv * G * D, V), generator=g) * 0.3).cuda()
    kd, vd, qd = kt.cuda(), vt.cuda(), qt.cuda()
    table = cas.PageTable(num_pages, PAGE)
    kp, vp = (torch.full((num_pages, PAGE, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pools, scale = cas.PagePools([kp, vp]), D ** -0.5
    r = np.random.default_rng(seed)

    def forward(problem, tokens):
        """One layer: append the tokens' keys and values, attend, project."""
        t = tokens.flatten().long()
        cas.paged_append(kd[t], vd[t], kp, vp, problem)
        q = qd[t]
        o = cas.paged_decode_fwd(q, kp, vp, None, None, None, Hkv, G, scale, problem=problem)[0] if decode else \
            cas.paged_chunk_fwd(q, kp, vp, problem)[0]
        return o, (o.float().flatten(1) @ wu).bfloat16()

    # A cartridge that all requests share, and a prompt of its own for each.
    toks = lambda n: torch.from_numpy(r.integers(0, V, n))
    cart = table.add(tokens=shared)
    cart_tokens = toks(shared)
    forward(table.problem([cart], [shared], Hkv, G, D, scale), cart_tokens.cuda()) if not decode else \
        cas.paged_append(kd[cart_tokens.cuda()], vd[cart_tokens.cuda()], kp, vp, table.problem([cart], [shared], Hkv, G, D, scale))
    seqs = [table.add([cart]) for _ in prompts]
    assert len(table.extend(seqs, prompts)) == 0
    prompt_tokens = [toks(n) for n in prompts]
    problem = table.problem(seqs, prompts, Hkv, G, D, scale)
    _, logits = forward(problem, torch.cat(prompt_tokens).cuda())
    last = np.cumsum(prompts) - 1
    logits = logits[torch.from_numpy(last).cuda()][:, None]
    before = table.info()
    search = cas.BeamSearch(table, pools, seqs, beams, end_token, steps)
    B = len(prompts)
    history, score, finished = [[[] for _ in range(beams)] for _ in range(B)], np.zeros((B, 1), np.float32), None
    while not search.done:
        logits[..., end_token] += bias
        seen = logits.float().cpu().double().numpy()
        tokens = search.step(logits)
        s, p, v = oracle.beam.select(seen, score, beams, finished, end_token)
        assert np.array_equal(tokens.cpu().numpy(), v)
        history = [[history[b][p[b, i]] + [int(v[b, i])] for i in range(beams)] for b in range(B)]
        fin = np.zeros((B, beams), bool) if finished is None else finished
        finished = np.stack([fin[b][p[b]] for b in range(B)]) | (v == end_token)
        got, score = search.results()
        assert got.cpu().numpy().tolist() == history
        score = score.cpu().numpy()
        assert np.allclose(score, s, rtol=2.0 ** -23, atol=6e-6) and np.array_equal(search.finished.cpu().numpy(), finished)
        if search.done:
            break
        problem = search.problem(Hkv, G, D, scale)
        o, logits = forward(problem, tokens)
        # every beam's keys, wherever they are
        lens, offs, ids = table.lists(search.seqs)
        k, w = kp.cpu(), vp.cpu()
        for b in range(B):
            for i in range(beams):
                n = b * beams + i
                want = torch.cat([cart_tokens, prompt_tokens[b], torch.tensor(history[b][i])])
                if finished[b, i]:
                    assert lens[n] == 1
                    continue
                at = torch.tensor(ids[offs[n]:offs[n + 1]])
                assert lens[n] == len(want)
                for pool, tab in ((k, kt), (w, vt)):
                    assert torch.equal(pool[at].reshape(-1, Hkv, D)[: len(want)], tab[want])
                K, W = (t_[want].double().numpy() for t_ in (kt, vt))
                q = qt[history[b][i][-1]].double().numpy()
                for h in range(Hkv * G):
                    a = K[:, h // G] @ q[h] * scale
                    e = np.exp(a - a.max())
                    ref = e @ W[:, h // G] / e.sum()
                    assert np.abs(o[n, h].double().cpu().numpy() - ref).max() <= 2e-2 * np.abs(ref).max()
        logits = logits.view(B, beams, V)
        # what the beams have in common is there once
        distinct = set(ids[: offs[len(search.seqs)]])
        assert table.info()["pages_used"] <= before["pages_used"] + len(distinct)
    search.close()
    assert table.info() == before
    with pytest.raises(RuntimeError):
        search.step(logits)
    return history


@pytest.mark.parametrize("beams,prompts,steps,bias,decode", [
    (4, [5], 20, -8.0, False), (4, [16, 31, 1], 20, 0.5, False), (8, [40, 17], 18, 1.0, True), (1, [3, 9], 12, -1.0, False),
    (16, [15], 5, -8.0, True), (3, [20, 21, 22, 23, 24], 9, 2.0, False),
])
def test_beam_search(gpu_lib, beams, prompts, steps, bias, decode):
    history = _run(gpu_lib, beams, prompts, steps, 7, bias, decode, seed=beams + steps)
    assert any(len(set(map(tuple, h))) > 1 for h in history) or beams == 1


def test_beam_search_out_of_pages(gpu_lib):
    """A step without enough free pages says so, and the search ends as it is."""
    import torch
    table = gpu_lib.PageTable(5, PAGE)
    pools = gpu_lib.PagePools([torch.zeros((5, PAGE, 1, 64), dtype=torch.bfloat16, device="cuda")])
    prompt = table.add(tokens=10)
    search = gpu_lib.BeamSearch(table, pools, [prompt], 8, 0, 4)
    with pytest.raises(gpu_lib.CasError) as e:
        search.step(torch.randn((1, 1, 100), device="cuda"))
    assert e.value.status == 8
    with pytest.raises(RuntimeError):
        search.step(torch.randn((1, 8, 100), device="cuda"))
    tokens, scores = search.results()
    assert tokens.shape == (1, 8, 1) and scores.shape == (1, 8)
    search.close()
    assert table.info()["pages_used"] == 1


def test_beam_search_refusals(gpu_lib):
    import torch
    table = gpu_lib.PageTable(20, PAGE)
    pool = torch.zeros((20, PAGE, 1, 64), dtype=torch.bfloat16, device="cuda")
    pools = gpu_lib.PagePools([pool])
    prompt = table.add(tokens=3)
    for args in (([prompt], 0, 0, 4), ([prompt], 2, 0, 0)):
        with pytest.raises(ValueError):
            gpu_lib.BeamSearch(table, pools, *args)
    with pytest.raises(ValueError):
        gpu_lib.BeamSearch(table, gpu_lib.PagePools([pool[:10]]), [prompt], 2, 0, 4)
    with pytest.raises(gpu_lib.CasError):
        gpu_lib.BeamSearch(table, pools, [prompt, 99], 2, 0, 4)
    assert table.info()["sequences"] == 1
    search = gpu_lib.BeamSearch(table, pools, [prompt], 2, 0, 4)
    with pytest.raises(RuntimeError):
        search.results()
    for shape in ((1, 2, 50), (2, 1, 50)):
        with pytest.raises(ValueError):
            search.step(torch.randn(shape, device="cuda"))
    search.step(torch.randn((1, 1, 50), device="cuda"))
    with pytest.raises(ValueError):
        search.step(torch.randn((1, 1, 50), device="cuda"))
    # fewer candidates than beams: the others go no further
    x = torch.full((1, 1, 50), float("-inf"), device="cuda")
    x[0, 0, 9] = 1.0
    search = gpu_lib.BeamSearch(table, pools, [prompt], 2, 0, 4)
    assert search.step(x).cpu()[0, 0] == 9 and not search.done
    assert search.scores.cpu()[0].tolist() == [0.0, float("-inf")] and search.table.lists(search.seqs)[0][:] == [4, 1]


def test_beam_search_in_pools_larger_than_the_table(gpu_lib):
    """The documented loop where the pools have pages that the table does not give out: those stay as they are."""
    import torch
    table = gpu_lib.PageTable(20, PAGE)
    kp, vp = (torch.full((33, PAGE, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pools, scale = gpu_lib.PagePools([kp, vp]), D ** -0.5
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    prompt = table.add(tokens=21)
    k, v = rand(21, Hkv, D), rand(21, Hkv, D)
    gpu_lib.paged_append(k, v, kp, vp, gpu_lib.DecodeProblem.from_tables([21], *table.lists([prompt]), 33, PAGE, Hkv, G, D, scale))
    search = gpu_lib.BeamSearch(table, pools, [prompt], 3, 0, 4)
    search.step(rand(1, 1, 50))
    while not search.done:
        k1, v1 = rand(3, Hkv, D), rand(3, Hkv, D)
        problem = search.problem(Hkv, G, D, scale)
        gpu_lib.paged_append(k1, v1, kp, vp, problem)
        o = gpu_lib.paged_chunk_fwd(rand(3, Hkv * G, D), kp, vp, problem)[0]
        assert bool(torch.isfinite(o).all())
        lens, offs, ids = table.lists(search.seqs)
        for i in range(3):
            at = torch.tensor(ids[offs[i]:offs[i + 1]], device="cuda")
            mine = kp[at].reshape(-1, Hkv, D)[:lens[i]]
            assert torch.equal(mine[-1], k1[i]) and (lens[i] == 1 or torch.equal(mine[:21], k))
        search.step(rand(1, 3, 50))
    assert bool((kp[20:] == 7.0).all()) and bool((vp[20:] == 7.0).all())
