"""GPU parity of beam selection and of the reordering of states against the
oracle in 64 bits.

Parents and tokens are equal. Scores are within half a step of fp32 relative to
the value (2^-24), plus the fp32 arithmetic of ln sum exp(x - b), b at most 16 below
the largest logit where what is below that counts. Relative to itself a term of argument
d = x - b is off by the rounding of d (|d| 2^-24), by a second one and a fourth of one for
log2 e where |b| is above 64 or so, or by a fourth of |x| 2^-24, |x| <= 80 + |d|, where it is not,
by one unit of the exponential instruction, 2^-23, and by eleven additions. Weighted by the terms'
share of the sum, |d| is at most ln V + 16 (the entropy of V tokens is at most ln V). For V up to 2^20
that is below (2.25 x 29.9 + 2 + 11) x 2^-24 = 4.8e-6 (or (1.25 x 29.9 + 20 + 13) x 2^-24).
States are equal in every bit.
"""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

INF = float("inf")
LSE_TOL = 4.8e-6


def _t():
    import torch
    return torch


def _dt(name):
    return _t().bfloat16 if name == "bf16" else _t().float32


def logits_of(B, N, V, dtype, seed, std=2.0, pad=0, shift=0):
    """[B, N, V] logits, a view of padded rows that begin `shift` elements into an allocation; what is around them would win."""
    t = _t()
    g = t.Generator().manual_seed(seed)
    flat = t.full((shift + B * N * (V + pad) + 8,), 1e5, dtype=_dt(dtype))
    x = flat[shift: shift + B * N * (V + pad)].view(B, N, V + pad)
    x[..., :V] = (t.randn((B, N, V), generator=g) * std).to(_dt(dtype))
    return flat, x[..., :V]


def on_gpu(flat, x):
    t = _t()
    d = flat.cuda()
    return t.as_strided(d, x.shape, x.stride(), x.storage_offset())


def check(cas, flat, x, scores, k, finished=None, pad_token=0, call=None):
    """beam_select against the oracle; returns what it gave."""
    t = _t()
    d = on_gpu(flat, x)
    f = None if finished is None else finished.cuda()
    got = (call or cas.beam_select)(d, scores.cuda(), k, finished=f, pad_token=pad_token)
    compare(got, x, scores, k, finished, pad_token)
    return got


def compare(got, x, scores, k, finished=None, pad_token=0):
    t = _t()
    s, p, v = (a.cpu().numpy() for a in got)
    rs, rp, rv = oracle.beam.select(x.double().numpy(), scores.double().numpy(), k, None if finished is None else finished.numpy(), pad_token)
    assert np.array_equal(p, rp) and np.array_equal(v, rv), (np.argwhere((p != rp) | (v != rv))[:4], p[:2], rp[:2], v[:2], rv[:2])
    fin = np.isfinite(rs)
    assert np.array_equal(np.isfinite(s), fin) and np.all(s[~fin] == -np.inf)
    tol = 2.0 ** -24 * np.abs(rs[fin]) + LSE_TOL
    if fin.any():
        assert np.all(np.abs(s[fin] - rs[fin]) <= tol), np.abs(s[fin] - rs[fin]).max()


def some_scores(B, N, seed):
    t = _t()
    return -3.0 - t.rand((B, N), generator=t.Generator().manual_seed(seed)) * 2


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,N,V,k,pad,shift", [
    (1, 1, 1, 1, 0, 0), (3, 1, 1, 1, 2, 1), (2, 2, 3, 6, 0, 1), (1, 4, 7, 8, 1, 3), (2, 3, 64, 5, 0, 0), (5, 2, 100, 64, 3, 5),
    (1, 64, 65, 64, 0, 7), (2, 1, 511, 1, 1, 2), (2, 5, 513, 10, 0, 0), (1, 3, 4095, 6, 0, 1), (2, 2, 4096, 4, 0, 0), (1, 2, 4097, 4, 7, 6),
    (2, 8, 8200, 16, 0, 0), (1, 2, 32000, 64, 0, 4), (3, 16, 10007, 32, 5, 1), (1, 4, 131073, 8, 3, 1), (40, 4, 1000, 8, 0, 0),
])
def test_select(gpu_lib, dtype, B, N, V, k, pad, shift):
    flat, x = logits_of(B, N, V, dtype, seed=V + k, pad=pad, shift=shift)
    check(gpu_lib, flat, x, some_scores(B, N, V), k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_select_a_large_vocabulary(gpu_lib, dtype):
    flat, x = logits_of(1, 2, 1 << 20, dtype, seed=3, shift=1)
    check(gpu_lib, flat, x, some_scores(1, 2, 3), 40)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [50, 4096, 20011])
@pytest.mark.parametrize("kind", ["constant", "zeros", "few values", "ascending", "descending", "one thread's", "one value above", "last",
                                  "subnormal", "spread"])
def test_select_orders(gpu_lib, dtype, V, kind):
    """Equal logits (the lowest tokens win), and orders of logits that no random row has."""
    t = _t()
    flat, x = logits_of(2, 3, V, dtype, seed=V, shift=3)
    i = t.arange(V)
    g = t.Generator().manual_seed(5)
    if kind == "constant":
        x[:] = 1.25
    elif kind == "zeros":
        x[:] = t.where(t.rand((2, 3, V), generator=g) < 0.5, 0.0, -0.0).to(x.dtype)
    elif kind == "few values":
        x[:] = t.randint(0, 4, (2, 3, V), generator=g).to(x.dtype)
    elif kind == "ascending":
        x[:] = (i * (8.0 / V)).to(x.dtype)
    elif kind == "descending":
        x[:] = (-i * (8.0 / V)).to(x.dtype)
    elif kind == "one thread's":
        x[:] += t.where(i // 8 % 64 == 5, 20.0, 0.0).to(x.dtype)
    elif kind == "one value above":
        x[:] = 0.0
        x[..., V // 2] = 3.0
        x[0, 1, V - 1] = 3.0
    elif kind == "last":
        x[..., -1] = 30.0
    elif kind == "subnormal":
        x[:] = (t.randint(-3, 4, (2, 3, V), generator=g) * 2.0 ** -130).to(x.dtype)
    else:
        x[:] = (t.randn((2, 3, V), generator=g) * 1e4).to(x.dtype)
    # Scores far enough apart for 64 bits, whatever the order of a sum is.
    scores = t.tensor([[-1.0, -1.7, -2.9], [-8.0, -1.3, -1.1]])
    check(gpu_lib, flat, x, scores, min(60, 3 * V))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [33, 9000])
def test_select_masks(gpu_lib, dtype, V):
    """Tokens at -inf or at the type's lowest value, rows that are left with few, one or no token, NaN and infinities,
    beams that have ended and scores that are none."""
    t = _t()
    B, N, k = 12, 6, 12
    flat, x = logits_of(B, N, V, dtype, seed=V, shift=1)
    low = t.finfo(x.dtype).min
    g = t.Generator().manual_seed(1)
    keep = t.rand((B, N, V), generator=g)
    x[0] = x[0].masked_fill(keep[0] < 0.9, -INF)
    x[1] = -INF
    x[1, 2, V // 3] = 1.0                              # one token in all
    x[2] = -INF                                        # none
    x[3] = x[3].masked_fill(keep[3] < 0.9, low)
    x[4] = low                                         # all at the lowest value: all alike
    x[5, 1, 7], x[5, 2, V - 1], x[5, 3, 0] = float("nan"), INF, INF
    x[5, 3, 1] = -INF
    x[6] = -INF
    x[6, 0] = float("nan")
    x[6, 3, [3, 30]] = -2.0
    x[7, :3] = -INF
    scores, finished = some_scores(B, N, V), t.zeros((B, N), dtype=t.bool)
    finished[8, [0, 3]] = True
    finished[9] = True
    finished[10, 1:] = True
    x[10, 1] = float("nan")                            # not looked at
    scores[7, 4], scores[8, 1], scores[8, 2] = -INF, INF, float("nan")
    scores[9, [1, 2]] = t.tensor([-INF, float("nan")])
    scores[11] = t.tensor([0.0] + [-INF] * (N - 1))    # a first step
    check(gpu_lib, flat, x, scores, k, finished, pad_token=V - 2)
    check(gpu_lib, flat, x, scores, 1, finished.to(t.uint8) * 3, pad_token=0)


def test_select_tells_near_scores_apart(gpu_lib):
    """Candidates of two beams whose scores are closer than 32 bits have them: 1e-9 to 1e-7 apart."""
    t = _t()
    for V in (70, 5000):
        for dtype in ("fp32", "bf16"):
            flat, x = logits_of(8, 4, V, dtype, seed=V)
            c = t.tensor([0.0, 2.0, -4.0, 8.0])[None, :, None]
            if dtype == "bf16":
                x[:, 0] = (x[:, 0].float() * 4).round().clamp(-16, 16).to(x.dtype) / 4
            else:
                x[:, 0] = (x[:, 0] * 1024).round() / 1024
            x[:] = (x[:, :1].float() + c).to(x.dtype)   # each beam's the first one's moved by a constant, exactly
            base = t.tensor([-0.01, -0.3, -1.0, -5.0, -20.0, -0.002, -0.7, -3.0])
            scores = base[:, None].repeat(1, 4)
            for i in range(4):
                for _ in range((3 * i) % 4):
                    scores[:, i] = t.nextafter(scores[:, i], t.tensor(0.0 if i % 2 else -100.0))
            check(gpu_lib, flat, x, scores, 16)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2048, 32000])
def test_select_equal_scores_around_64(gpu_lib, dtype, V):
    """Constant rows and random ones that differ by a constant, around logits of +-64, where the sums' terms change their
    form: equal scores go by beam, whatever the sums are off by."""
    t = _t()
    shifts = t.tensor([[-64.0, 64.0], [64.0, -64.0], [-63.5, 63.5], [-64.0, 63.5], [-65.0, 64.0], [64.0, 65.0], [-64.5, -63.5],
                       [62.0, -66.0]])[..., None]
    k = min(40, 2 * V)
    flat, x = logits_of(8, 2, V, dtype, seed=V)
    x[:] = shifts.to(x.dtype)
    check(gpu_lib, flat, x, t.full((8, 2), -2.5), k)
    step = 1.0 if dtype == "bf16" else 2.0 ** -10   # (both types hold such sums)
    base = (3 * t.randn((8, 1, V), generator=t.Generator().manual_seed(V)) / step).round() * step
    x[:] = (base + shifts.round()).to(x.dtype)
    check(gpu_lib, flat, x, t.full((8, 2), -2.5), k)


@pytest.mark.parametrize("V", [2, 1000])
def test_select_scores_a_few_1e_13_apart(gpu_lib, V):
    """Beam 0's logits are all 0; beam 1 has 0 and V - 1 times d, and a score that puts it 2e-13 to 4e-13 ahead by the
    definition. The sums of the second pass are to be exact enough for that."""
    t = _t()
    found = {2: ["-0x1.4394a4p-7 -0x1.42c824p-8", "-0x1.5d1d2ep-7 -0x1.5c2f22p-8", "-0x1.3cc734p-7 -0x1.3c0336p-8",
                 "-0x1.479916p-7 -0x1.46c77ap-8", "-0x1.58801cp-7 -0x1.579850p-8", "-0x1.5ab608p-7 -0x1.59cb40p-8"],
             1000: ["-0x1.53b9eep-7 -0x1.536282p-7", "-0x1.47dab4p-7 -0x1.47865ap-7", "-0x1.5822bap-7 -0x1.57ca2ap-7",
                    "-0x1.3d2fe0p-7 -0x1.3cde48p-7", "-0x1.46fa64p-7 -0x1.46a644p-7", "-0x1.52ca3cp-7 -0x1.52730ep-7"]}[V]
    d, own = t.tensor([[float.fromhex(h) for h in pair.split()] for pair in found], dtype=t.float64).unbind(1)
    flat, x = logits_of(len(found), 2, V, "fp32", seed=V)
    x[:, 0] = 0.0
    x[:, 1, 0], x[:, 1, 1:] = 0.0, d[:, None].float()
    ahead = own - (((V - 1) * d.exp() + 1) / V).log()   # (64 bits hold these to 1e-15)
    assert bool((x[:, 1, 1].double() == d).all()) and bool(((ahead > 2e-13) & (ahead < 4e-13)).all())
    scores = t.stack([t.zeros_like(own), own], 1).float()
    got = check(gpu_lib, flat, x, scores, 2)
    assert got[1][:, 0].tolist() == [1] * len(found)


def test_select_near_scores_of_rising_rows(gpu_lib):
    """Logits that rise along the row, as far as the sums keep what they began with and a little further, in beams that
    differ by a constant and a few steps of fp32 in their scores."""
    t = _t()
    for dtype, chunk in (("fp32", 2048), ("bf16", 4096)):
        for rise in (15.5, 16.0, 16.5, 40.0):
            flat, x = logits_of(6, 4, 3 * chunk, dtype, seed=chunk)
            x[:, 0, :512] = 0.0
            x[:, 0, 512: chunk] = 15.5
            x[:, 0, chunk: 2 * chunk] = rise
            x[:, 0, 2 * chunk:] = rise + 16.5
            x[:, 0, 7 * chunk // 3:] = rise + 0.5
            x[:] = (x[:, :1].float() + t.tensor([0.0, 64.0, -32.0, 8.0])[None, :, None]).to(x.dtype)
            scores = t.tensor([-0.01, -0.3, -1.0, -5.0, -20.0, -0.002])[:, None].repeat(1, 4)
            for i in range(4):
                for _ in range((3 * i) % 4):
                    scores[:, i] = t.nextafter(scores[:, i], t.tensor(0.0 if i % 2 else -100.0))
            check(gpu_lib, flat, x, scores, 12)


@pytest.mark.parametrize("rise", [15.5, 16.5, 40.0])
def test_select_near_scores_of_long_rising_rows(gpu_lib, rise):
    """As above in rows so long that a wave has several chunks of them."""
    t = _t()
    flat, x = logits_of(2, 4, 2048 * 2048, "fp32", seed=9, std=0.0)
    row = x[0, 0].view(1024, 2, 2048)   # (of the chunks, every second one)
    row[:, 0, 512:] = 15.5
    row[:, 1] = rise
    x[:] = row.reshape(-1) + t.tensor([0.0, 64.0, -32.0, 8.0])[None, :, None]
    scores = t.tensor([[-0.3], [-5.0]]).repeat(1, 4)
    for i in range(4):
        for _ in range((3 * i) % 4):
            scores[:, i] = t.nextafter(scores[:, i], t.tensor(0.0 if i % 2 else -100.0))
    check(gpu_lib, flat, x, scores, 12)


def test_select_equal_beams(gpu_lib):
    """Beams alike in every bit: equal scores go by beam, then token. Rows of odd length begin at different alignments."""
    t = _t()
    for dtype in ("fp32", "bf16"):
        for V in (64, 5001, 12345):
            flat, x = logits_of(3, 5, V, dtype, seed=V, shift=1)
            x[:] = x[:, 2:3].clone()
            scores = t.tensor([[-2.5], [-1e-3], [-700.0]]).repeat(1, 5)
            check(gpu_lib, flat, x, scores, 32)


@pytest.mark.parametrize("N,V,k", [(9, 700, 30), (12, 20011, 50), (40, 5001, 64), (64, 300, 64), (64, 20000, 64)])
def test_select_many_equal_beams(gpu_lib, N, V, k):
    """Many beams alike, with random logits and with constant ones (masses of equal candidates), some of them a little better."""
    t = _t()
    for dtype in ("fp32", "bf16"):
        flat, x = logits_of(2, N, V, dtype, seed=V, shift=1)
        x[:] = x[:, 2:3].clone()
        x[1] = 0.25
        scores = t.full((2, N), -2.5)
        scores[0, N // 2] = t.nextafter(t.tensor(-2.5), t.tensor(0.0))
        scores[1, 3] = t.nextafter(t.tensor(-2.5), t.tensor(-9.0))
        check(gpu_lib, flat, x, scores, k)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,V,k", [(20, 20000, 50), (33, 8191, 33), (64, 40000, 64), (17, 100000, 40), (8, 300000, 64)])
def test_select_many_beams(gpu_lib, dtype, N, V, k):
    flat, x = logits_of(2, N, V, dtype, seed=V + k, shift=2)
    check(gpu_lib, flat, x, some_scores(2, N, V), k)


@pytest.mark.parametrize("seed", range(6))
def test_select_random(gpu_lib, seed):
    t = _t()
    r = np.random.default_rng(seed)
    B, N, V = int(r.integers(1, 9)), int(r.integers(1, 20)), int(np.exp(r.uniform(0, 10)))
    k = int(r.integers(1, min(64, N * V) + 1))
    flat, x = logits_of(B, N, V, r.choice(["bf16", "fp32"]), seed, std=float(r.choice([0.1, 1, 5])), pad=int(r.integers(0, 9)),
                        shift=int(r.integers(0, 9)))
    x.masked_fill_(t.rand(x.shape, generator=t.Generator().manual_seed(seed)) < r.choice([0, 0.3, 0.999]), -INF)
    finished = t.rand((B, N), generator=t.Generator().manual_seed(seed)) < r.choice([0, 0.3])
    check(gpu_lib, flat, x, some_scores(B, N, seed), k, finished, pad_token=int(r.integers(0, V)))


def test_select_streams_outs_and_workspace(gpu_lib):
    """Another stream than the current one, the caller's outputs and workspace, a second call on them."""
    t = _t()
    side = t.cuda.Stream()
    flat, x = logits_of(3, 4, 7001, "bf16", 1)
    flat2, x2 = logits_of(3, 4, 7001, "bf16", 2)
    scores = some_scores(3, 4, 1)
    d, d2, s = on_gpu(flat, x), on_gpu(flat2, x2), scores.cuda()
    n = gpu_lib.beam_select_workspace_size(d, 8)
    ws = t.full((n,), 255, dtype=t.uint8, device="cuda")
    outs = [t.full((3, 8), 7, dtype=dt, device="cuda") for dt in (t.float32, t.int32, t.int32)]
    side.wait_stream(t.cuda.current_stream())
    got = gpu_lib.beam_select(d2, s, 8, outs=outs, stream=side, workspace=ws)
    got = gpu_lib.beam_select(d, s, 8, outs=outs, stream=side, workspace=ws)
    side.synchronize()
    assert all(a is b for a, b in zip(got, outs))
    compare(got, x, scores, 8)
    with pytest.raises(gpu_lib.CasError):
        gpu_lib.beam_select(d, s, 8, workspace=ws[: n - 256])
    with pytest.raises(TypeError):
        gpu_lib.beam_select(d, s, 8, outs=outs[::-1])


def test_select_at_once(gpu_lib):
    """Two calls at once, on two streams with workspaces of their own."""
    t = _t()
    streams, made = [t.cuda.Stream() for _ in range(2)], []
    inputs = [logits_of(4, 8, 30011, "bf16", i) for i in range(2)]
    scores = some_scores(4, 8, 1)
    dev = [on_gpu(*i) for i in inputs]
    s = scores.cuda()
    t.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            made.append((i, gpu_lib.beam_select(dev[i], s, 16, stream=streams[i])))
    t.cuda.synchronize()
    for i, got in made:
        compare(got, inputs[i][1], scores, 16)


def test_select_and_reorder_in_a_graph(gpu_lib):
    """A captured step, replayed on new logits with eager work between the replays."""
    t = _t()
    B, N, V = 3, 4, 9001
    flat, x = logits_of(B, N, V, "bf16", 1)
    d, scores = on_gpu(flat, x), some_scores(B, N, 2)
    s, hist = scores.cuda(), t.arange(B * N * 33, dtype=t.int32, device="cuda").view(B, N, 33)
    outs = [t.empty((B, N), dtype=dt, device="cuda") for dt in (t.float32, t.int32, t.int32)]
    y = t.empty_like(hist)
    ws = t.empty(gpu_lib.beam_select_workspace_size(d, N), dtype=t.uint8, device="cuda")
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        gpu_lib.beam_select(d, s, N, outs=outs, workspace=ws)
        gpu_lib.beam_reorder([hist], outs[1], outs=[y])
    for i in range(4):
        _, xi = logits_of(B, N, V, "bf16", 10 + i)
        d.copy_(xi)
        hist += 1
        eager = gpu_lib.beam_select(d, s, N)
        graph.replay()
        t.cuda.synchronize()
        compare(outs, xi, scores, N)
        assert all(t.equal(a, b) for a, b in zip(eager, outs))
        assert np.array_equal(y.cpu().numpy(), oracle.beam.reorder(hist.cpu().numpy(), outs[1].cpu().numpy()))


def test_select_rows_past_four_gib(gpu_lib):
    """A row stride that puts the last beam 4 GiB behind the first: offsets of 64 bits."""
    t = _t()
    V, stride = 5003, (1 << 30) + 24
    flat, x = logits_of(1, 4, V, "bf16", 4)
    big = t.empty(3 * stride + V, dtype=t.bfloat16, device="cuda")
    d = t.as_strided(big, (1, 4, V), (4 * stride, stride, 1))
    d.copy_(x)
    scores = some_scores(1, 4, 4)
    compare(gpu_lib.beam_select(d, scores.cuda(), 8), x, scores, 8)


@pytest.mark.parametrize("B,N,V", [(70001, 2, 9), (1 << 18, 4, 3), (300, 1, 4099)])
def test_select_many_entries(gpu_lib, B, N, V):
    """More batch entries than a grid's second dimension has, up to the most rows."""
    t = _t()
    flat, x = logits_of(B, N, V, "fp32", seed=B, shift=1)
    scores = some_scores(B, N, 4)
    s, p, v = (a.cpu() for a in gpu_lib.beam_select(on_gpu(flat, x), scores.cuda(), 3))
    ref = (scores.double()[..., None] + t.log_softmax(x.double(), -1)).view(B, N * V)
    best, at = ref.sort(dim=1, descending=True, stable=True)
    assert t.equal(p, (at[:, :3] // V).int()) and t.equal(v, (at[:, :3] % V).int())
    assert bool(((s - best[:, :3]).abs() <= 2.0 ** -24 * best[:, :3].abs() + LSE_TOL).all())


# -- reordering ---------------------------------------------------------------
def states(B, N, shape, dtype, seed):
    """Integers that every type holds."""
    t = _t()
    x = t.randint(0, 120, (B, N, *shape), dtype=t.int32, generator=t.Generator().manual_seed(seed))
    return x.to({"uint8": t.uint8, "int16": t.int16, "bf16": t.bfloat16, "int32": t.int32, "float64": t.float64}[dtype])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,N,shape,dtype", [(1, 1, (1,), "uint8"), (2, 4, (), "int32"), (3, 8, (777,), "int32"), (2, 3, (5,), "uint8"),
                                             (2, 5, (31,), "int16"), (1, 16, (8, 3, 64), "bf16"), (4, 17, (40,), "float64"),
                                             (2, 64, (1000,), "bf16"), (70, 2, (9,), "float64"), (2, 33, (3, 7), "uint8"), (0, 4, (5,), "int32"),
                                             (70001, 2, (9,), "uint8"), (1 << 18, 4, (3,), "int32"),
                                             (2, 4, (0,), "int32"), (1, 6, (200003,), "uint8")])
def test_reorder(gpu_lib, B, N, shape, dtype, in_place):
    t = _t()
    x = states(B, N, shape, dtype, 1)
    parents = t.randint(0, N, (B, N), dtype=t.int32, generator=t.Generator().manual_seed(2))
    d = x.cuda()
    y, = gpu_lib.beam_reorder([d], parents.cuda(), outs=[d] if in_place else None)
    if B:
        ref = oracle.beam.reorder(x.double().numpy(), parents.numpy())
        assert np.array_equal(y.cpu().double().numpy(), ref)
    assert y.dtype == x.dtype and (y is d) == in_place
    if not in_place:
        assert t.equal(d.cpu(), x)


@pytest.mark.parametrize("shift", [0, 1, 2, 4, 8])
def test_reorder_slices_and_several(gpu_lib, shift):
    """Used parts of longer states at any alignment, several tensors in one call, more beams out than in; what lies
    around the rows stays as it is."""
    t = _t()
    B, N, M = 3, 4, 7
    parents = t.randint(0, N, (B, M), dtype=t.int32, generator=t.Generator().manual_seed(shift))
    xs, ys, refs = [], [], []
    for i, (cap, used) in enumerate(((64, 33), (100, 100), (48, 1), (4096, 4001), (200, 0))):
        x = states(B, N, (cap + shift + 16,), "uint8", i).cuda()[:, :, shift:shift + used]
        y = t.full((B, M, cap + 2 * shift + 5), 99, dtype=t.uint8, device="cuda")
        xs.append(x)
        ys.append(y)
        refs.append(oracle.beam.reorder(x.cpu().numpy(), parents.numpy()))
    views = [y[:, :, 2 * shift: 2 * shift + x.shape[2]] for x, y in zip(xs, ys)]
    gpu_lib.beam_reorder(xs, parents.cuda(), outs=views)
    for x, y, ref in zip(xs, ys, refs):
        h, n = y.cpu().numpy(), x.shape[2]
        assert np.array_equal(h[:, :, 2 * shift: 2 * shift + n], ref)
        assert (h[:, :, : 2 * shift] == 99).all() and (h[:, :, 2 * shift + n:] == 99).all()


def test_reorder_parents_out_of_range(gpu_lib):
    """Rows without a parent in range stay as they were."""
    t = _t()
    x = states(2, 4, (50,), "int32", 1)
    parents = t.tensor([[0, -1, 4, 3], [1 << 30, 2, -(1 << 31), 2]], dtype=t.int32)
    ok = (parents >= 0) & (parents < 4)
    ref = t.where(ok[:, :, None], t.from_numpy(oracle.beam.reorder(x.numpy(), parents.clamp(0, 3).numpy())), x)
    d = x.cuda()
    gpu_lib.beam_reorder([d], parents.cuda(), outs=[d])
    assert t.equal(d.cpu(), ref)
    y = x.cuda().clone()
    gpu_lib.beam_reorder([x.cuda()], parents.cuda(), outs=[y])
    assert t.equal(y.cpu(), ref)


def test_reorder_interleaved_states(gpu_lib):
    """Keys and values of beams in one tensor, reordered in place in one call."""
    t = _t()
    x = states(3, 5, (2, 40), "int32", 1)
    d, parents = x.cuda(), t.randint(0, 5, (3, 5), dtype=t.int32)
    k, v = d[:, :, 0], d[:, :, 1]
    gpu_lib.beam_reorder([k, v], parents.cuda(), outs=[k, v])
    assert np.array_equal(d.cpu().numpy(), oracle.beam.reorder(x.numpy(), parents.numpy()))


def test_reorder_past_four_gib(gpu_lib):
    t = _t()
    stride = (1 << 31) + 64
    big = t.zeros(2 * stride + 1000, dtype=t.uint8, device="cuda")
    x = t.as_strided(big, (1, 3, 777), (0, stride, 1))
    h = states(1, 3, (777,), "uint8", 3)
    x.copy_(h)
    parents = t.tensor([[2, 0, 1]], dtype=t.int32)
    gpu_lib.beam_reorder([x], parents.cuda(), outs=[x])
    assert np.array_equal(x.cpu().numpy(), oracle.beam.reorder(h.numpy(), parents.numpy()))
