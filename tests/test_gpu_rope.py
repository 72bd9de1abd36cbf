"""GPU parity of the rotary positions and of appending to the paged cache
against the oracle in extended precision.

Tolerance, per element: half a step of the output's type relative to the value
(bf16 2^-8, fp32 2^-24), plus the fp32 arithmetic before that rounding, relative
to the pair's length r: cos and sin are within 1.6e-7 (the reduced angle's
rounding 3e-8, the series and its roundings 1e-7, the factor 3e-8), so each of
the two products is off by 1.6e-7 of its channel, sqrt(2) 1.6e-7 r together, and
their roundings and the sum's add 2 x 2^-24 r: below 2^-21 r = 4.8e-7 r.
Values that are not rotated, and every row of a pool that is not written, are
equal in every bit.
"""
import ctypes

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def _t():
    import torch
    return torch


def _dt(name):
    return _t().bfloat16 if name == "bf16" else _t().float32


def _rand(shape, dtype, seed):
    t = _t()
    g = t.Generator().manual_seed(seed)
    return t.randn(shape, generator=g).to(_dt(dtype))


def _host(x):
    return x.detach().cpu().double().numpy()


def check(y, x, pos, rope, dtype, inverse=False):
    """y against the oracle's rotation of x ([tokens, heads, d] both)."""
    x, y, n = _host(x), _host(y), rope.rotary_dim // 2
    il = rope.layout == "interleaved"
    scale = float(np.float32(rope.scale))
    ref = oracle.rope.rotate(x, pos, rope.turns, scale, il, inverse)
    tol = EPS[dtype] * np.abs(ref) + 2.0 ** -21 * scale * oracle.rope.pair_norms(x, n, il) + 1e-38
    tol[..., 2 * n:] = 0.0
    bad = np.abs(y - ref) > tol
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), np.abs(y - ref).max())


def bits(x):
    return x.contiguous().view(_t().int16 if x.dtype == _t().bfloat16 else _t().int32)


def _positions(T, seed, hi=1 << 20):
    r = np.random.default_rng(seed)
    p = r.integers(-hi, hi, T).astype(np.int32)
    p[: min(T, 3)] = [0, hi - 1, -hi][: min(T, 3)]
    return p


# -- rope ---------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,heads,D,R", [(1, (1,), 64, 64), (1, (32, 8), 128, 128), (137, (6, 2), 128, 64), (33, (5,), 64, 16),
                                         (1027, (4, 1, 3), 64, 48), (2050, (40, 8), 128, 112)])
def test_rope(gpu_lib, T, heads, D, R, dtype, layout):
    t = _t()
    rope = gpu_lib.Rope(R, 1e4, layout=layout, scaling=gpu_lib.RopeScaling("by_parts", 4.0, 4096))
    pos = _positions(T, T)
    xs = [_rand((T, h, D), dtype, 10 + i).cuda() for i, h in enumerate(heads)]
    dpos = t.from_numpy(pos).cuda()
    keep = [x.clone() for x in xs]
    for inverse, call in ((False, gpu_lib.rope_fwd), (True, gpu_lib.rope_bwd)):
        ys = call(xs, dpos, rope)
        for x, y, k in zip(xs, ys, keep):
            check(y, x, pos, rope, dtype, inverse)
            assert t.equal(x, k)
    # the same in place
    zs = gpu_lib.rope_bwd(xs, dpos, rope, outs=xs)
    for z, y, x in zip(zs, ys, xs):
        assert z is x and t.equal(bits(z), bits(y))


def test_rope_strides(gpu_lib):
    """Slices of one projection, out of place and in place, head-major storage,
    a head that several share, and leading dimensions: the same bits."""
    t = _t()
    B, S, Hq, Hkv, D = 2, 70, 6, 2, 128
    rope = gpu_lib.Rope(D, 1e6)
    pos = _positions(B * S, 3)
    dpos = t.from_numpy(pos).cuda()
    x = _rand((B, S, Hq + 2 * Hkv, D), "bf16", 5).cuda()
    q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
    yq, yk = gpu_lib.rope_fwd([q, k], dpos.view(B, S), rope)
    assert yq.shape == q.shape and yq.is_contiguous()
    check(yq.view(B * S, Hq, D), q.reshape(B * S, Hq, D), pos, rope, "bf16")
    check(yk.view(B * S, Hkv, D), k.reshape(B * S, Hkv, D), pos, rope, "bf16")
    # head-major in and out
    xh = q.reshape(B * S, Hq, D).permute(1, 0, 2).contiguous().permute(1, 0, 2)
    yh = t.full((Hq, B * S, D), float("nan"), dtype=t.bfloat16, device="cuda").permute(1, 0, 2)
    gpu_lib.rope_fwd([xh], dpos, rope, outs=[yh])
    assert t.equal(bits(yh), bits(yq.view(B * S, Hq, D)))
    # one head read by all
    one = x[:, :, :1].expand(B, S, Hq, D)
    y1, = gpu_lib.rope_fwd([one], dpos, rope)
    assert t.equal(bits(y1), bits(yq[:, :, :1].expand(B, S, Hq, D)))
    # one token's vector read at every position
    tok = x[:1, :1, :2].reshape(1, 2, D).expand(B * S, 2, D)
    y2, = gpu_lib.rope_fwd([tok], dpos, rope)
    check(y2, tok, pos, rope, "bf16")
    # in place on the slices; the values between them stay
    v = x[:, :, Hq + Hkv:].clone()
    gpu_lib.rope_fwd([q, k], dpos, rope, outs=[q, k])
    assert t.equal(bits(q), bits(yq)) and t.equal(bits(k), bits(yk)) and t.equal(bits(x[:, :, Hq + Hkv:]), bits(v))


def test_rope_gradient(gpu_lib):
    """<dy, R x> = <R^T dy, x>, and differences: R is linear, so (R(x + h e) - R x) / h
    is column e at any h (fp32: 2^-21 of the pair on each side of the difference)."""
    t = _t()
    T, D, R = 3, 64, 32
    pos = np.array([5, 70000, -9], dtype=np.int32)
    dpos = t.from_numpy(pos).cuda()
    for layout in ("half", "interleaved"):
        rope = gpu_lib.Rope(R, 1e4, layout=layout, scale=1.3)
        x, dy = _rand((T, 1, D), "fp32", 1).cuda(), _rand((T, 1, D), "fp32", 2).cuda()
        dx, = gpu_lib.rope_bwd([dy], dpos, rope)
        y0, = gpu_lib.rope_fwd([x], dpos, rope)
        for c in range(D):
            xe = x.clone()
            xe[:, :, c] += 1.0
            ye, = gpu_lib.rope_fwd([xe], dpos, rope)
            want = (dy.double() * (ye.double() - y0.double())).sum(-1)
            # |x|, |x + e| < 6 in a pair of length < 9; 2 channels of dy (< 5) see a difference, the others none
            assert (want - dx[:, :, c].double()).abs().max().item() <= 2 * 2 * 5 * 9 * 1.3 * 2.0 ** -21


def test_rope_far_positions_and_special_values(gpu_lib):
    """The ends of int32; NaN and infinities reach their own pair and nothing else."""
    t = _t()
    D, R = 64, 32
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 12345678], dtype=np.int32)
    rope = gpu_lib.Rope(R, 1e4)
    x = _rand((4, 2, D), "fp32", 8)
    y, = gpu_lib.rope_fwd([x.cuda()], t.from_numpy(pos).cuda(), rope)
    ref = oracle.rope.rotate(_host(x), pos, rope.turns)
    # 2^31 positions: the double product of 3.4e8 turns is off by 2 x 2^-53 of them, 5e-7 radians at most
    assert np.abs(_host(y) - ref).max() <= 4.8 * (5e-7 + 2.0 ** -21)
    z = x.clone()
    z[0, 0, 3] = float("nan")
    z[1, 1, 40] = float("inf")    # not rotated
    z[2, 0, 17] = float("-inf")   # pair 1
    w, = gpu_lib.rope_fwd([z.cuda()], t.from_numpy(pos).cuda(), rope)
    w, y = w.cpu(), y.cpu()
    assert t.isnan(w[0, 0, [3, 19]]).all() and w[1, 1, 40] == float("inf") and not t.isfinite(w[2, 0, [1, 17]]).any()
    for i, h, cs in ((0, 0, [3, 19]), (1, 1, [40]), (2, 0, [1, 17])):
        w[i, h, cs] = y[i, h, cs]
    assert t.equal(w, y)


def test_rope_in_a_graph_and_on_a_stream(gpu_lib):
    t = _t()
    rope = gpu_lib.Rope(128, 1e6)
    x, pos = _rand((40, 4, 128), "bf16", 1).cuda(), t.arange(40, dtype=t.int32, device="cuda")
    y = t.empty_like(x)
    rope.device_turns(x.device)
    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    z, = gpu_lib.rope_fwd([x], pos, rope, stream=s)
    s.synchronize()
    check(z, x, np.arange(40), rope, "bf16")
    # (a rope that is dropped at once, on another stream than its own)
    outs = [gpu_lib.rope_fwd([x], pos, gpu_lib.Rope(128, 1e6 + i), stream=s)[0] for i in range(8)]
    s.synchronize()
    for i, z in enumerate(outs):
        check(z, x, np.arange(40), gpu_lib.Rope(128, 1e6 + i), "bf16")
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        gpu_lib.rope_fwd([x], pos, rope, outs=[y])
    for i in range(3):
        x.copy_(_rand((40, 4, 128), "bf16", 20 + i))
        pos += 1000
        g.replay()
        want, = gpu_lib.rope_fwd([x], pos, rope)
        t.cuda.synchronize()
        assert t.equal(bits(y), bits(want))


def test_rope_past_4_gib(gpu_lib):
    """Offsets past 32 bits: 5 tokens 2^30 elements apart."""
    t = _t()
    rope = gpu_lib.Rope(64, 1e4)
    base = t.zeros((4 << 30) + 256, dtype=t.bfloat16, device="cuda")
    x = t.as_strided(base, (5, 2, 64), (1 << 30, 64, 1))
    x.copy_(_rand((5, 2, 64), "bf16", 3))
    pos = np.array([1, 2, 3, 4, 5], dtype=np.int32)
    y, = gpu_lib.rope_fwd([x], t.from_numpy(pos).cuda(), rope)
    check(y, x, pos, rope, "bf16")
    z = x.clone()
    gpu_lib.rope_fwd([x], t.from_numpy(pos).cuda(), rope, outs=[x])
    assert t.equal(bits(x), bits(y)) and z.shape == x.shape


# -- append -------------------------------------------------------------------
def _problem(cas, q, kv, P, Hkv, g, D, seed, spare=3):
    """Requests with private pages in shuffled order."""
    r = np.random.default_rng(seed)
    need = [-(-L // P) for L in kv]
    ids = r.permutation(sum(need) + spare).tolist()
    pages = [[ids.pop() for _ in range(n)] for n in need]
    npages = sum(need) + spare
    return pages, npages, cas.DecodeProblem(q, kv, pages, npages, P, Hkv, g, D, 0.125)


def _append_case(cas, q, kv, P, Hkv, g, D, R, layout, seed, fused=True, pad=0, starts=None, pages=None, with_q=True):
    t = _t()
    if pages is None:
        pages, npages, prob = _problem(cas, q, kv, P, Hkv, g, D, seed)
    else:
        npages = 1 + max(p for pl in pages for p in pl)
        prob = cas.DecodeProblem(q, kv, pages, npages, P, Hkv, g, D, 0.125)
    T, Hq = sum(q), Hkv * g
    rope = cas.Rope(R, 1e4, layout=layout, scaling=cas.RopeScaling("linear", 2.0)) if R else None
    x = _rand((T + pad, Hq + 2 * Hkv, D), "bf16", seed).cuda()
    qq, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        qq, k, v = qq.contiguous(), k.permute(1, 0, 2).contiguous().permute(1, 0, 2), v.contiguous()
    kp, vp = (_rand((npages, P, Hkv, D), "bf16", seed + i).cuda() for i in (1, 2))
    kp0, vp0 = kp.clone(), vp.clone()
    q_out = t.full((T + pad, Hq, D), 7.0, dtype=t.bfloat16, device="cuda")
    got = cas.paged_append(k, v, kp, vp, prob, rope=rope, q=qq if with_q else None, q_out=q_out if with_q else None, starts=starts)
    pos = np.concatenate([np.arange(n) + (L - n if starts is None else s)
                          for n, L, s in zip(q, kv, starts or [0] * len(q))] + [np.empty(0)]).astype(np.int32)
    dpos = t.from_numpy(pos).cuda()
    if rope is not None and T:
        want, = cas.rope_fwd([k[:T]], dpos, rope)
        check(want, k[:T], pos, rope, "bf16")
    else:
        want = k[:T].clone()
    if with_q and T:
        assert got is q_out
        check(q_out[:T], qq[:T], pos, rope, "bf16")
        assert t.equal(bits(q_out[:T]), bits(cas.rope_fwd([qq[:T]], dpos, rope)[0]))
    assert (q_out[T:] == 7.0).all()
    ek, ev = oracle.rope.append(bits(kp0).cpu().numpy(), bits(vp0).cpu().numpy(), bits(want).cpu().numpy(),
                                bits(v).cpu().numpy(), q, kv, pages)
    assert np.array_equal(bits(kp).cpu().numpy(), ek) and np.array_equal(bits(vp).cpu().numpy(), ev)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("Hkv,g,D,R,layout", [(8, 4, 128, 128, "half"), (1, 1, 64, 16, "interleaved"), (3, 5, 128, 80, "half")])
def test_append(gpu_lib, P, Hkv, g, D, R, layout):
    _append_case(gpu_lib, [1, 40, 0, 17, 129, 3], [1, 77, 5, 17, 129 + 250, 64], P, Hkv, g, D, R, layout, P + D)
    _append_case(gpu_lib, [1, 1, 1], [1, 16, 129], P, Hkv, g, D, R, layout, P, fused=False, pad=5)


def test_append_variants(gpu_lib):
    A = lambda *a, **k: _append_case(gpu_lib, *a, **k)
    A([2, 5], [9, 40], 16, 2, 2, 64, 64, "half", 1, starts=[100000, -3])
    A([2, 5], [9, 40], 16, 2, 2, 64, 0, "half", 2, with_q=False)             # no rotation
    A([2, 5], [9, 40], 16, 2, 2, 64, 64, "half", 3, with_q=False)
    A([0, 0], [9, 0], 16, 2, 2, 64, 64, "half", 4, pad=2)                     # nothing to write
    A([2000], [2100], 16, 2, 4, 128, 128, "half", 5, pages=[list(range(132))])          # consecutive pages
    A([700, 1], [700, 20], 16, 1, 1, 64, 64, "half", 6, pages=[list(range(43, -1, -1)), [50, 44]])
    A([1] * 300, [17 + i for i in range(300)], 32, 2, 1, 64, 32, "interleaved", 7)       # more requests than one launch holds
    A([9] * 260, [9 + i for i in range(260)], 16, 2, 1, 128, 128, "half", 8)
    for D, P in ((64, 16), (128, 32), (64, 128)):
        # sixteen tokens to a workgroup, that begin and end inside pages; one request over several launches
        A([700, 3, 341, 1], [707, 40, 341 + 11, 5], P, 2, 3, D, 32, "half", 9 + D)
        A([300, 5], [309, 7], P, 1, 2, D, 16, "interleaved", 10 + D, pad=1)
    A([12000, 5, 9000], [12003, 5, 9000 + 29], 16, 1, 1, 64, 64, "half", 11)


def test_append_past_4_gib(gpu_lib):
    """Pages past 4 GiB of the pools (2^21 bytes each, the last of 2,600)."""
    t = _t()
    P, Hkv, D, n = 128, 64, 128, 2600
    kp = t.zeros((n, P, Hkv, D), dtype=t.bfloat16, device="cuda")
    vp = t.zeros_like(kp)
    prob = gpu_lib.DecodeProblem([3, 1], [130, 5], [[2, n - 1], [n - 2]], n, P, Hkv, 1, D, 0.1)
    x = _rand((4, Hkv, D), "bf16", 1).cuda()
    gpu_lib.paged_append(x, -x, kp, vp, prob)
    for i, (p, r) in enumerate([(2, 127), (n - 1, 0), (n - 1, 1), (n - 2, 4)]):
        assert t.equal(kp[p, r], x[i]) and t.equal(vp[p, r], -x[i])
        kp[p, r] = 0
        vp[p, r] = 0
    assert not kp.any() and not vp.any()


def test_append_in_a_graph(gpu_lib):
    t = _t()
    rope = gpu_lib.Rope(64, 1e4)
    pages, n, prob = _problem(gpu_lib, [3, 1], [20, 33], 16, 2, 2, 64, 1)
    k, v, q = (_rand((4, h, 64), "bf16", h).cuda() for h in (2, 3, 4))
    v = v[:, :2]
    kp, vp = (t.zeros((n, 16, 2, 64), dtype=t.bfloat16, device="cuda") for _ in range(2))
    out = gpu_lib.paged_append(k, v, kp, vp, prob, rope=rope, q=q)
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        gpu_lib.paged_append(k, v, kp, vp, prob, rope=rope, q=q, q_out=out)
    for i in range(3):
        k.copy_(_rand((4, 2, 64), "bf16", 50 + i))
        q.copy_(_rand((4, 4, 64), "bf16", 60 + i))
        kp.zero_()
        vp.zero_()
        out.zero_()
        g.replay()
        k2, v2 = t.zeros_like(kp), t.zeros_like(vp)
        want = gpu_lib.paged_append(k, v, k2, v2, prob, rope=rope, q=q)
        t.cuda.synchronize()
        assert t.equal(bits(kp), bits(k2)) and t.equal(bits(vp), bits(v2)) and t.equal(bits(out), bits(want)) and kp.any()


def test_append_q_in_place(gpu_lib):
    t = _t()
    rope = gpu_lib.Rope(64, 1e4)
    pages, n, prob = _problem(gpu_lib, [3, 1], [20, 33], 16, 2, 2, 64, 1)
    k, q = _rand((4, 2, 64), "bf16", 1).cuda(), _rand((4, 4, 64), "bf16", 2).cuda()
    kp, vp = (t.zeros((n, 16, 2, 64), dtype=t.bfloat16, device="cuda") for _ in range(2))
    want = gpu_lib.paged_append(k, k, kp, vp, prob, rope=rope, q=q)
    assert gpu_lib.paged_append(k, k, kp, vp, prob, rope=rope, q=q, q_out=q) is q and t.equal(bits(q), bits(want))


def test_training_step_with_positions(gpu_lib):
    """rope_fwd, prefix attention and back: the gradients of the unrotated queries
    and keys against the oracle's, whose rotation is applied in 64 bits (bars of
    the attention: 2e-2 of the largest value; the rotated inputs are rounded to
    bf16 once on each side)."""
    t = _t()
    B, S, Hkv, g, D, C = 2, 40, 2, 2, 64, 50
    rope = gpu_lib.Rope(D, 1e4)
    pos = np.tile(np.arange(S) + C, B).astype(np.int32)
    dpos = t.from_numpy(pos).cuda()
    q, k, v, do = (_rand((B, S, h, D), "bf16", i).cuda() for i, h in enumerate((Hkv * g, Hkv, Hkv, Hkv * g)))
    ck, cv = (_rand((C, Hkv, D), "bf16", 9 + i).cuda() for i in range(2))
    dck, dcv = t.empty_like(ck), t.empty_like(cv)
    rows = [[gpu_lib.Segment(ck, cv, dck, dcv)]] * B
    sc = 0.125
    qr, kr = gpu_lib.rope_fwd([q, k], dpos, rope)
    o, lse = gpu_lib.prefix_attn_fwd(qr, kr, v, rows, Hkv, g, sc)
    dqr, dkr, dv = gpu_lib.prefix_attn_bwd(qr, kr, v, rows, Hkv, g, sc, o, lse, do)
    dq, dk = gpu_lib.rope_bwd([dqr, dkr], dpos, rope)
    rot = lambda x, inv=False: oracle.rope.rotate(x.reshape(B * S, -1, D), pos, rope.turns, inverse=inv).reshape(x.shape)
    bf = lambda a: t.from_numpy(a).to(t.bfloat16).double().numpy()
    args = (bf(rot(_host(q))), bf(rot(_host(k))), _host(v), [_host(ck)], [_host(cv)], [[0]] * B, sc, g)
    O, LSE = oracle.forward(*args)
    rdq, rdk, rdv, rdc, _ = oracle.backward(*args, _host(do), O=O, LSE=LSE)
    for got, want in ((o, O), (dq, rot(rdq, True)), (dk, rot(rdk, True)), (dv, rdv), (dck, rdc[0])):
        assert np.abs(_host(got) - want).max() <= 2e-2 * np.abs(want).max()
