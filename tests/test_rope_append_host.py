"""Rotary positions and appending to the paged cache without a GPU: the oracle's
pins, the frequency formulas, and every refusal (argument checks run before any
HIP call, so made-up addresses stand in for device memory)."""
import ctypes
import math

import numpy as np
import pytest

import oracle


@pytest.fixture(scope="module")
def cas():
    import paper_2606_04557_amd as cas
    cas.load()
    return cas


@pytest.fixture(scope="module")
def L():
    from paper_2606_04557_amd import _lib
    return _lib


# -- the oracle ---------------------------------------------------------------
@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotation_pins(interleaved):
    r = np.random.default_rng(1)
    x, pos, turns = r.normal(size=(5, 2, 12)), np.array([0, 1, -3, 700, 2 ** 30]), [0.31, 0.02, 1e-4, 0.5]
    y = oracle.rope.rotate(x, pos, turns, 1.0, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 8:], x[..., 8:])
    # complex multiplication, by pairs
    for i, f in enumerate(turns):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, 4 + i)
        for t in range(4):
            z = (x[t, :, p] + 1j * x[t, :, q]) * np.exp(2j * np.pi * pos[t] * f)
            assert np.allclose(y[t, :, p] + 1j * y[t, :, q], z, rtol=0, atol=1e-12)
    # the score of two rotated vectors depends on the distance of their positions
    a, b = x[:1], x[1:2]
    dot = lambda s, t: (oracle.rope.rotate(a, [s], turns, 1.0, interleaved) * oracle.rope.rotate(b, [t], turns, 1.0, interleaved)).sum()
    assert abs(dot(5, 9) - dot(105, 109)) < 1e-12
    # the inverse undoes it, and is its transpose
    s = 1.25
    assert np.allclose(oracle.rope.rotate(y, pos, turns, 1.0, interleaved, True), x, atol=1e-12)
    dy = r.normal(size=x.shape)
    lhs = (dy * oracle.rope.rotate(x, pos, turns, s, interleaved)).sum()
    rhs = (oracle.rope.rotate(dy, pos, turns, s, interleaved, True) * x).sum()
    # (the copied channels are not scaled, in either direction)
    assert abs(lhs - rhs) < 1e-11


def test_oracle_append_pins():
    k = np.arange(4.0).reshape(4, 1, 1) + 10
    kp, vp = oracle.rope.append(np.zeros((3, 2, 1, 1)), np.ones((3, 2, 1, 1)), k, -k, [3, 0, 1], [4, 2, 2], [[2, 0], [1], [1]])
    assert kp[:, :, 0, 0].tolist() == [[11, 12], [0, 13], [0, 10]] and vp[2, 1, 0, 0] == -10 and vp[1, 0, 0, 0] == 1


# -- frequencies --------------------------------------------------------------
def test_frequencies(cas):
    R, base = 64, 5e5
    f = [base ** (-2.0 * i / R) / (2 * math.pi) for i in range(R // 2)]
    near = lambda a, b: np.allclose(a, b, rtol=1e-14, atol=0)
    assert near(cas.Rope(R, base).turns, f) and cas.Rope(R, base).scale == 1.0
    assert near(cas.Rope(R, base, scaling=cas.RopeScaling("linear", 8)).turns, [x / 8 for x in f])
    ntk = cas.Rope(R, base, scaling=cas.RopeScaling("ntk", 4)).turns
    assert near(ntk[0], f[0]) and near(ntk[-1], f[-1] / 4)      # the slowest pair is interpolated, the fastest kept
    parts = cas.Rope(R, base, scaling=cas.RopeScaling("by_parts", 4, 8192, 1, 4))
    assert parts.scale == 0.1 * math.log(4) + 1
    for a, x in zip(parts.turns, f):
        n = 8192 * x                                             # turns within the original length
        w = 0.0 if n <= 1 else 1.0 if n >= 4 else (n - 1) / 3
        assert near(a, (1 - w) * x / 4 + w * x)
    assert any(1 < 8192 * x < 4 for x in f)
    assert cas.Rope(R, base, scaling=cas.RopeScaling("by_parts", 4, 8192, 1, 4, attention_factor=1.0)).scale == 1.0
    assert cas.Rope(R, base, scaling=cas.RopeScaling("by_parts", 0.5, 8192)).scale == 1.0
    own = cas.Rope(32, frequencies=[0.25] * 16, scale=2.0)
    assert near(own.turns, [0.25 / (2 * math.pi)] * 16) and own.scale == 2.0


@pytest.mark.parametrize("make", [
    lambda c: c.Rope(24), lambda c: c.Rope(0), lambda c: c.Rope(144), lambda c: c.Rope(64, base=0.0),
    lambda c: c.Rope(64, base=float("nan")), lambda c: c.Rope(64, scaling=c.RopeScaling("linear", 0.0)),
    lambda c: c.Rope(64, scaling=c.RopeScaling("by_parts", 4, 0.0)),
    lambda c: c.Rope(64, scaling=c.RopeScaling("by_parts", 4, 4096, 32, 32)),
])
def test_frequency_refusals(cas, make):
    with pytest.raises(cas.CasError):
        make(cas)


def test_binding_refusals(cas):
    import torch
    with pytest.raises(ValueError):
        cas.Rope(64, layout="other")
    with pytest.raises(ValueError):
        cas.Rope(64, scaling=cas.RopeScaling("dynamic", 2))
    with pytest.raises(ValueError):
        cas.Rope(64, frequencies=[1.0] * 31)
    rope, pos = cas.Rope(64), torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 2, 64)
    for xs, p in (([], pos), ([x] * 5, pos), ([x], pos[:3]), ([x, torch.zeros(3, 2, 64)], pos), ([x, x.to(torch.bfloat16)], pos),
                  ([torch.zeros(4, 64)], pos), ([torch.zeros(4, 2, 128)[..., ::2]], pos), ([x], pos.repeat(2)[::2]),
                  ([torch.zeros(2, 3, 2, 64)[:, :2]], pos),              # no common token stride
                  ([x], pos)):                                             # not on a GPU
        with pytest.raises(ValueError):
            cas.rope_fwd(xs, p, rope)
    with pytest.raises(TypeError):
        cas.rope_fwd([x], pos.long(), rope)
    with pytest.raises(TypeError):
        cas.rope_fwd([x.half()], pos, rope)
    with pytest.raises(ValueError):
        cas.rope_fwd([x], pos, rope, outs=[torch.zeros(4, 2, 65)])
    prob = cas.DecodeProblem([2, 1], [2, 17], [[0], [1, 2]], 4, 16, 2, 2, 64, 0.125)
    bf = torch.bfloat16
    kp = torch.zeros(4, 16, 2, 64, dtype=bf)
    k, q = torch.zeros(3, 2, 64, dtype=bf), torch.zeros(3, 4, 64, dtype=bf)
    ok = dict(k=k, v=k, k_pages=kp, v_pages=kp, problem=prob, rope=rope, q=q)
    for over in (dict(k=k[:2]), dict(v=torch.zeros(3, 3, 64, dtype=bf)), dict(k_pages=kp[:3]), dict(q=q[:, :3]),
                 dict(v_pages=torch.zeros(4, 16, 2, 128, dtype=bf)[..., :64]), dict(starts=[1]), dict(q_out=q[:2]), {}):
        with pytest.raises(ValueError):                                    # ({}: not on a GPU)
            cas.paged_append(**{**ok, **over})
    with pytest.raises(TypeError):
        cas.paged_append(**{**ok, "k": k.float()})
    with pytest.raises(OverflowError):
        cas.paged_append(**{**ok, "starts": [0, 1 << 31]})


# -- refusals of the library ---------------------------------------------------
A = 1 << 40   # addresses that are never touched
INVALID, UNSUPPORTED, ALIGN = 1, 2, 3


def rope_call(cas, L, tokens=10, D=128, dtype=0, positions=A, n=1, inverse=0, rope=None, tensors=None, **over):
    r = L.Rope(0, 64, A + (1 << 20), 1.0)
    for k, v in (rope or {}).items():
        setattr(r, k, v)
    base = dict(x=2 * A, y=3 * A, x_stride_tok=256, x_stride_head=128, y_stride_tok=256, y_stride_head=128, heads=2)
    ts = (L.RopeTensor * 4)(*[L.RopeTensor(**{**base, **t}) for t in (tensors or [over])])
    return cas.load().cas_rope(ctypes.byref(r), dtype, D, tokens, positions, ts, n if not tensors else len(tensors), inverse, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(tokens=-1), INVALID), (dict(tokens=(1 << 24) + 1), UNSUPPORTED),
    (dict(n=0), INVALID), (dict(n=5), INVALID), (dict(positions=None), INVALID), (dict(positions=A + 2), ALIGN),
    (dict(rope=dict(layout=2)), INVALID), (dict(rope=dict(rotary_dim=8)), UNSUPPORTED), (dict(rope=dict(rotary_dim=40)), UNSUPPORTED),
    (dict(rope=dict(rotary_dim=144)), UNSUPPORTED), (dict(rope=dict(turns=None)), INVALID), (dict(rope=dict(turns=A + 4)), ALIGN),
    (dict(rope=dict(scale=0.0)), INVALID), (dict(rope=dict(scale=float("nan"))), INVALID),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(heads=0), INVALID), (dict(x=2 * A + 8), ALIGN), (dict(y=3 * A + 2), ALIGN),
    (dict(x_stride_tok=260), ALIGN), (dict(y_stride_head=132), ALIGN), (dict(x_stride_tok=-256), INVALID),
    (dict(x_stride_tok=1 << 32), INVALID),
    (dict(y_stride_tok=0), INVALID), (dict(y_stride_head=0), INVALID), (dict(y_stride_tok=128), INVALID),       # y overlaps itself
    (dict(y=2 * A + 16), INVALID), (dict(y=2 * A, x_stride_tok=512), INVALID),                                   # y over x
    (dict(y=A - 256 * 20 + 128), INVALID), (dict(y=A + (1 << 20)), INVALID),                                     # over positions, turns
    (dict(tensors=[{}, dict(x=4 * A)]), INVALID),                                                                # two outputs in one place
    (dict(tensors=[{}, dict(x=3 * A + 512, y=5 * A)]), INVALID),                                                 # y over another x
    # slices of one buffer whose rows overlap by a head
    (dict(tensors=[dict(x_stride_tok=512, y=2 * A, y_stride_tok=512), dict(x=2 * A + 256, y=2 * A + 256, x_stride_tok=512,
                                                                           y_stride_tok=512)]), INVALID),
])
def test_rope_refusals(cas, L, kw, code):
    assert rope_call(cas, L, **kw) == code, cas.load().cas_last_error_message()
    assert cas.load().cas_last_error_message()


def test_rope_of_no_tokens_is_nothing(cas, L):
    assert rope_call(cas, L, tokens=0, positions=None, x=None, y=None) == 0


def problem(cas, q, kv, pages, npages=16, P=16, Hkv=2, g=2, D=64):
    return cas.DecodeProblem(q, kv, pages, npages, P, Hkv, g, D, 0.125)


def append_plan_status(cas, prob):
    lib, h = cas.load(), ctypes.c_void_p()
    s = lib.cas_paged_append_plan_create(ctypes.byref(prob.c), ctypes.byref(h))
    assert (s == 0) == bool(h)
    if h:
        assert lib.cas_paged_append_plan_matches(h, ctypes.byref(prob.c)) == 1
        lib.cas_paged_append_plan_destroy(h)
    return s


@pytest.mark.parametrize("q,kv,pages,code", [
    ([1, 1], [17, 33], [[0, 1], [0, 2, 3]], 0),                       # a shared whole page is only read
    ([0, 1], [16, 17], [[0], [0, 1]], 0),                             # a request without new tokens
    ([0, 0], [0, 5], [[], [3]], 0),                                   # nothing at all to write
    ([16, 1], [16, 17], [[1], [1, 0]], INVALID),                      # a shared page is written
    ([1, 1], [16, 16], [[5], [5]], INVALID),                          # the same row twice
    ([1, 1], [4, 3], [[5], [5]], INVALID),                            # one writes row 3, the other reads rows 0..2 and writes row 2
    ([1, 0], [4, 3], [[5], [5]], 0),                                  # row 3 is written, rows 0..2 are shared
    ([1, 0], [4, 4], [[5], [5]], INVALID),                            # row 3 is written and read
    ([1, 1], [4, 4], [[5], [5 + 3]], 0),
    ([1], [40], [[1, 2, 1]], INVALID),                                # a request that reads its own last page twice
    ([20], [40], [[0, 1, 0]], INVALID),
    ([3], [2], [[0]], INVALID), ([1], [17], [[0]], INVALID), ([1], [1], [[16]], INVALID), ([1], [1], [[-1]], INVALID),
    ([-1], [4], [[0]], INVALID),
])
def test_append_tables(cas, q, kv, pages, code):
    assert append_plan_status(cas, problem(cas, q, kv, pages)) == code, cas.load().cas_last_error_message()


def test_append_far_page_ids_with_equal_low_bits(cas):
    """Pages 5 and 5 + 2^16 share the bits that pass over unwritten pages."""
    big = (1 << 16) + 5
    assert append_plan_status(cas, problem(cas, [1, 1], [4, 30], [[5], [big, 6]], npages=1 << 17)) == 0
    assert append_plan_status(cas, problem(cas, [1, 1], [4, 30], [[big], [big, 6]], npages=1 << 17)) == INVALID


@pytest.mark.parametrize("field,value,code", [
    ("batch", 0, INVALID), ("num_kv_heads", 0, INVALID), ("group_size", 0, INVALID), ("head_dim", 80, UNSUPPORTED),
    ("page_size", 48, UNSUPPORTED), ("num_pages", 0, INVALID), ("q_offsets", None, INVALID), ("page_ids", None, INVALID),
    ("num_kv_heads", 1 << 16, UNSUPPORTED),
])
def test_append_problem_fields(cas, field, value, code):
    prob = problem(cas, [1], [4], [[5]])
    setattr(prob.c, field, value)
    assert append_plan_status(cas, prob) == code


def append_call(cas, L, rope=True, k_pages=8 * A, v_pages=9 * A, starts=None, **over):
    prob = problem(cas, [2, 0, 1], [18, 7, 1], [[0, 1], [2], [3]])
    t = L.Append(k=2 * A, v=3 * A, k_stride_tok=128, k_stride_head=64, v_stride_tok=128, v_stride_head=64, q=4 * A,
                 q_stride_tok=256, q_stride_head=64, q_out=5 * A)
    for k, v in over.items():
        setattr(t, k, v)
    if starts:
        t.starts = (ctypes.c_int32 * 3)(*starts)
    r = L.Rope(0, 64, A, 1.0)
    return cas.load().cas_paged_append(ctypes.byref(prob.c), ctypes.byref(r) if rope else None, ctypes.byref(t), k_pages, v_pages, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rope=False), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k_pages=None), INVALID),
    (dict(q_out=None), INVALID), (dict(k=2 * A + 2), ALIGN), (dict(q_out=5 * A + 8), ALIGN), (dict(v_pages=9 * A + 4), ALIGN),
    (dict(k_stride_tok=132), ALIGN), (dict(v_stride_head=-64), INVALID), (dict(q_stride_head=4), ALIGN),
    (dict(v_pages=8 * A + 64), INVALID), (dict(k=8 * A), INVALID), (dict(q_out=9 * A), INVALID), (dict(q=5 * A + 128), INVALID),
    (dict(q_out=A - 64), INVALID), (dict(q=4 * A, q_out=4 * A, q_stride_tok=512), INVALID),
    (dict(starts=[(1 << 31) - 2, 0, 0]), INVALID),
])
def test_append_refusals(cas, L, kw, code):
    assert append_call(cas, L, **kw) == code, cas.load().cas_last_error_message()


def test_append_plan_arguments(cas, L):
    lib = cas.load()
    prob = problem(cas, [1], [4], [[5]])
    assert lib.cas_paged_append_plan_create(ctypes.byref(prob.c), None) == INVALID
    assert lib.cas_paged_append_plan_create(None, ctypes.byref(ctypes.c_void_p())) == INVALID
    assert lib.cas_paged_append_run(None, None, ctypes.byref(L.Append()), None, None, None) == INVALID
    plan = prob.append_plan()
    assert prob.append_plan() is plan
    prob._kv[0] = 5                                                   # the table changes: planned again
    assert prob.append_plan() is not plan
