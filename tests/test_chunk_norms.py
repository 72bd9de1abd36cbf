"""The chunk attention's error as a whole: its norm over a request against the
norm that its roundings give, which shows what a bar for every element lets pass
(one key's wrong value row among a thousand moves each element by less than that
bar).

The bar. A value m 2^e (1 <= m < 2) rounded to bf16 is off by at most 2^-8 2^e, by
any amount up to that with equal chance: 2^-16 / 3 of its square in the mean,
taken at m = 1. Every weight p_j and every element of O is rounded once, each for
itself, so
  E |o - O|^2 <= 2^-16 / 3 (|O|^2 + sum_j p_j^2 |v_j|^2)
summed over rows, where m spread over [1, 2) makes the left side about 0.54 of the
right (the mean of 1 / m^2 for a logarithmic spread is 3 / (8 ln 2)). The rest is
room for chance: |e|^2 of one rounding has a deviation of 0.9 of its mean, so sums
of 64 independent ones and more stay below 0.54 (1 + 5 x 0.9 / 8) = 0.85 of the
right side at five deviations; requests of fewer rows are taken together. fp32
errors (2^-17 of a weight) do not count beside that.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")


def squares(o, q, K, V, n, scale, g):
    """(|o - O|^2, the bar) of one request's n new tokens, over all heads; K and V: [L, Hkv, d] in 64 bits."""
    L = K.shape[0]
    see = torch.arange(L, device=K.device)[None, :] <= torch.arange(L - n, L, device=K.device)[:, None]
    err = bar = 0.0
    for h in range(q.shape[1]):
        S = (q[:, h].double() @ K[:, h // g].T * scale).masked_fill(~see, -np.inf)
        p = torch.softmax(S, 1)
        O = p @ V[:, h // g]
        err += ((o[:, h].double() - O) ** 2).sum().item()
        bar += 2.0 ** -16 / 3 * ((O ** 2).sum() + ((p ** 2) @ (V[:, h // g] ** 2).sum(1)).sum()).item()
    return err, bar


def check_norms(o, q, kp, vp, counts, kv, pages, scale, g):
    few = [0.0, 0.0, 0]
    t0 = 0
    for n, L, pl in zip(counts, kv, pages):
        if n:
            ids = torch.tensor(pl, device=kp.device)
            K, V = (x[ids].reshape(-1, *x.shape[2:])[:L].double() for x in (kp, vp))
            err, bar = squares(o[t0: t0 + n], q[t0: t0 + n], K, V, n, scale, g)
            rows = n * q.shape[1]
            if rows >= 64:
                assert err <= bar, (n, L, err / bar)
            else:
                few = [few[0] + err, few[1] + bar, few[2] + rows]
        t0 += n
    if few[2] >= 64:
        assert few[0] <= few[1], few


def rounded_attention(q, K, V, scale, g):
    """Attention in fp32 whose weights and result are rounded to bf16, in torch."""
    n, L = q.shape[0], K.shape[0]
    see = torch.arange(L)[None, :] <= torch.arange(L - n, L)[:, None]
    out = torch.empty(q.shape, dtype=torch.bfloat16)
    for h in range(q.shape[1]):
        S = (q[:, h].float() @ K[:, h // g].float().T * scale).masked_fill(~see, -np.inf)
        e = torch.exp(S - S.amax(1, keepdim=True))
        out[:, h] = (e.to(torch.bfloat16).float() @ V[:, h // g].float() / e.sum(1, keepdim=True)).to(torch.bfloat16)
    return out


@pytest.mark.parametrize("n,L", [(64, 64), (50, 1000), (64, 2000)])
def test_the_bar_shows_one_wrong_value_row(n, L):
    """On the CPU: attention with those roundings stays below 0.85 of the bar; with
    one key's values exchanged for another's in the definition it is above it."""
    gen = torch.Generator().manual_seed(n + L)
    rand = lambda *s: torch.randn(s, generator=gen).to(torch.bfloat16)
    q, K, V = rand(n, 4, 64), rand(L, 2, 64), rand(L, 2, 64)
    o = rounded_attention(q, K, V, 0.125, 2)
    err, bar = squares(o, q, K.double(), V.double(), n, 0.125, 2)
    assert 0.25 * bar < err < 0.85 * bar, err / bar
    wrong = V.double().clone()
    wrong[3] = wrong[5]                                   # (keys that every query sees)
    err, bar = squares(o, q, K.double(), wrong, n, 0.125, 2)
    assert err > bar, err / bar


@pytest.mark.gpu
@pytest.mark.parametrize("P,D,Hkv,g", [(16, 128, 8, 4), (32, 64, 4, 3), (128, 128, 2, 5), (64, 64, 1, 8)])
def test_norms(gpu_lib, P, D, Hkv, g):
    """Blocks of 256 rows, whole and in pieces, narrow ones, requests in a few rows,
    single tokens, with and without shared cartridges."""
    import test_gpu_chunk as chunk
    b = 256 // g
    for counts, kv, carts, cart_pages in (
            ([1, b - 1, b, 0, b + 1, 5, 1, 2 * b + 3], [1, b - 1, b + 64, 9, b + 127, 64, 65, 2 * b + 3 + 1000], (), 0),
            ([33], [5000], (), 0), ([700, 20, 3], [2900, 1500, 4000], (), 0),
            ([1] * 40, [4 * 512 + 1 + 3 * i for i in range(40)], [[0, 1, 2, 3]] * 40, 512 // P),
            ([1] * 20 + [70, 300] + [1] * 20, [2 * 512 + 400 + 3 * i for i in range(42)], [[i % 2, 2] for i in range(42)], 512 // P)):
        _, q, kp, vp, o, lse, pages = chunk.run(gpu_lib, counts, kv, P, Hkv, g, D, seed=P + D + g, carts=carts, cart_pages=cart_pages)
        check_norms(o, q, kp, vp, counts, kv, pages, float(np.float32(D ** -0.5)), g)


@pytest.mark.gpu
def test_serving_steps_closely(gpu_lib):
    """Prompts prefilled in chunks and then decoded: every step's rotated queries and
    keys against the oracle's rotation, element by element, and its attention against
    the definition on the very bits that are in q and the pages, with the bars of a
    single call for O, LSE and the norm."""
    import test_gpu_chunk as chunk
    import test_gpu_rope as rope_tests
    Hkv, g, D, P, cart = 2, 4, 128, 16, 64
    Hq, scale = Hkv * g, float(np.float32(D ** -0.5))
    rope = gpu_lib.Rope(D, 1e4)
    steps = [[100, 20], [48, 15], [1, 1], [1, 1]]
    own = [[4 + 2 * j for j in range(10)], [5 + 2 * j for j in range(10)]]
    kp, vp = (torch.zeros((24, P, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kp[:4], vp[:4] = (chunk._rand((4, P, Hkv, D), s, i) for i, s in ((1, 0.7), (2, 1.0)))
    done = [0, 0]
    for i, counts in enumerate(steps):
        kv = [cart + d + n for d, n in zip(done, counts)]
        pages = [([0, 1, 2, 3] + o)[: -(-L // P)] for o, L in zip(own, kv)]
        prob = gpu_lib.DecodeProblem(counts, kv, pages, 24, P, Hkv, g, D, scale)
        x = chunk._rand((sum(counts), Hq + 2 * Hkv, D), 1.0, 10 + i)
        q = gpu_lib.paged_append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], kp, vp, prob, rope=rope, q=x[:, :Hq])
        pos = np.concatenate([np.arange(L - n, L) for n, L in zip(counts, kv)]).astype(np.int32)
        rope_tests.check(q, x[:, :Hq], pos, rope, "bf16")
        slot = [(pl[j // P], j % P) for n, L, pl in zip(counts, kv, pages) for j in range(L - n, L)]
        at = [torch.tensor(s, device="cuda") for s in zip(*slot)]
        rope_tests.check(kp[at[0], at[1]], x[:, Hq:Hq + Hkv], pos, rope, "bf16")
        assert torch.equal(vp[at[0], at[1]], x[:, Hq + Hkv:])
        o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
        chunk.compare(o, lse, q, kp, vp, counts, kv, pages, scale, g)
        check_norms(o, q, kp, vp, counts, kv, pages, scale, g)
        done = [d + n for d, n in zip(done, counts)]
