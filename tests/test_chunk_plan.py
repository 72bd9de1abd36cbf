"""The chunk attention's launch plan and refusals (host only): every row of
every KV head walks each 64-key tile it sees exactly once, pieces have places of
their own, and nothing is listed that has no rows."""
import ctypes
import random

import pytest

TILE, ROWS = 64, 256
A = 1 << 40   # addresses that are never touched
INVALID, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 5


@pytest.fixture(scope="module")
def cas():
    import paper_2606_04557_amd as cas
    cas.load()
    return cas


def problem(cas, q, kv, P=16, Hkv=2, g=2, D=64, pages=None):
    pages = pages or [[j for j in range(-(-L // P))] for L in kv]
    npages = 1 + max((p for pl in pages for p in pl), default=0)
    return cas.DecodeProblem(q, kv, pages, npages, P, Hkv, g, D, 0.125)


def check(cas, q, kv, **kw):
    prob = problem(cas, q, kv, **kw)
    P, Hkv, g = prob.c.page_size, prob.c.num_kv_heads, prob.c.group_size
    info, wgs = cas.chunk_plan(prob)
    items = [i for w in wgs for i in w]
    assert len(wgs) == info.workgroups and len(items) == info.items and sum(i[7] - i[6] for i in items) == info.key_tiles
    # Blocks of one size (the largest of them: 256, or what a half of it holds).
    rows = next((r for r in (32, 64, 128) if all(i[10] - i[4] <= r for i in items) and all(i[4] % r == 0 for i in items) and
                 all(i[10] == min(i[1] * g, i[4] + r) for i in items)), ROWS)
    seen, parts = {}, {}
    granule0, at = {}, 0
    listed = {i[0] for i in items}
    for b, L in enumerate(kv):
        if q[b] and sum(q[:b]) in listed:
            granule0[b], at = at, at + -(-(-(-L // P) * (P // 16)) // 4) * 4
    first = {sum(q[:b]): b for b in reversed(range(len(q))) if q[b]}
    for tok0, n, L, pg, row0, kvh, t0, t1, part, _, row1 in items:
        b = first[tok0]
        assert row1 == min(n * g, row0 + rows)
        assert (n, L, pg) == (q[b], kv[b], granule0[b]) and row0 % rows == 0 and row0 < n * g and 0 <= kvh < Hkv
        last = L - n + (row1 - 1) // g      # of the block's rows
        assert 0 <= t0 < t1 <= last // TILE + 1
        seen.setdefault((b, row0, kvh), []).append((t0, t1, last // TILE + 1))
        parts.setdefault((b, row0, kvh), []).append(part)
    want = {(b, r, k) for b, n in enumerate(q) for r in range(0, n * g, rows) for k in range(Hkv)}
    gone = {b for b, _, _ in want - set(seen)}                     # requests that the decode kernels take
    assert set(seen) == {w for w in want if w[0] not in gone} and all(q[b] == 1 for b in gone) and len(gone) == info.decode_tokens
    all_parts = []
    for k, v in seen.items():
        v.sort()
        assert v[0][0] == 0 and v[-1][1] == v[-1][2] and all(a[1] == b[0] for a, b in zip(v, v[1:])) and len(v) <= info.max_partials
        p = sorted(parts[k])
        assert p == [-1] if len(p) == 1 else p == list(range(p[0], p[0] + len(p))) and p[0] >= 0
        all_parts += [x for x in p if x >= 0]
    assert sorted(all_parts) == list(range(info.partials))
    assert cas.paged_chunk_workspace_size(prob) == info.ws_bytes >= info.partials * rows * (prob.c.head_dim + 1) * 4
    return info


def test_plans(cas):
    r = random.Random(4)
    for _ in range(150):
        B = r.randint(1, 12)
        q = [r.choice([0, 1, 1, r.randint(1, 60), r.randint(1, 900)]) for _ in range(B)]
        kv = [n + r.choice([0, r.randint(0, 100), r.randint(0, 20000)]) for n in q]
        check(cas, q, kv, P=r.choice([16, 32, 64, 128]), Hkv=r.choice([1, 2, 3, 4, 8, 12, 16]), g=r.choice([1, 2, 3, 5, 8]),
              D=r.choice([64, 128]))


def loads(cas, prob):
    info, wgs = cas.chunk_plan(prob)
    return info, [sum(i[7] - i[6] for i in w) for w in wgs]


def test_workgroups_have_equal_shares(cas):
    """A prompt's chunk over a long context is cut into one workgroup per compute
    unit, blocks that fill them without a rest are not cut, and neither are many."""
    kw = dict(Hkv=8, g=4, D=128)
    one, n = loads(cas, problem(cas, [512], [16384 + 512], **kw))
    assert one.workgroups == 256 and max(n) <= 1.1 * one.key_tiles / 256
    full, n = loads(cas, problem(cas, [2048] * 4, [4096] * 4, **kw))
    assert full.partials == 0
    odd, n = loads(cas, problem(cas, [300] * 16, [4500] * 16, **kw))       # 640 blocks: two and a half per unit
    assert odd.workgroups == 256 and odd.partials > 0 and max(n) <= 1.1 * odd.key_tiles / 256
    many, n = loads(cas, problem(cas, [2000] * 16, [4500] * 16, **kw))
    assert many.partials == 0 and many.workgroups == many.items
    assert loads(cas, problem(cas, [1], [64], **kw))[0].partials == 0


def test_shared_single_tokens_go_to_the_decode_kernels(cas):
    """Runs of single-token requests that read the same cartridges, and only those."""
    kw = dict(Hkv=8, g=4, D=128)
    carts = [list(range(64 * c, 64 * c + 64)) for c in range(16)]
    nxt = iter(range(1024, 9999))

    def req(cs, own):
        return [p for c in cs for p in carts[c]] + [next(nxt) for _ in range(-(-own // 16))], len(cs) * 1024 + own

    shared = [req(range(8), 5 + i) for i in range(20)]
    alone = [req([], 4000) for _ in range(20)]
    chunk = [req([0, 1], 300)]
    def info(reqs, q):
        return check(cas, q, [L for _, L in reqs], pages=[p for p, _ in reqs], **kw)
    i = info(shared, [1] * 20)
    assert (i.decode_parts, i.decode_tokens, i.workgroups) == (1, 20, 0)
    assert info(alone, [1] * 20).decode_parts == 0
    i = info(shared[:10] + chunk + shared[10:] + alone, [1] * 10 + [300] + [1, 0] * 5 + [1] * 20)
    assert i.decode_parts in (1, 2) and 10 <= i.decode_tokens <= 35 and i.workgroups > 0
    assert info(shared, [2] * 20).decode_parts == 0
    assert info(shared[:1], [1]).decode_parts == 0
    assert check(cas, [1] * 20, [L for _, L in shared], pages=[p for p, _ in shared], Hkv=1, g=40, D=64).decode_parts == 0


def test_heads_keep_to_their_xcds(cas):
    """Workgroup i runs on XCD i mod 8."""
    for Hkv in (1, 2, 4, 8, 16):
        _, wgs = cas.chunk_plan(problem(cas, [700, 1, 90], [5000, 3000, 90], Hkv=Hkv, g=4, D=128))
        groups = min(Hkv, 8)
        for i, w in enumerate(wgs):
            assert all(x[5] % groups == i % groups for x in w)


@pytest.mark.parametrize("q,kv,pages,code", [
    ([0], [0], [[]], 0), ([1], [1], [[0]], 0), ([2], [1], [[0]], INVALID), ([-1], [1], [[0]], INVALID), ([1], [17], [[0]], INVALID),
    ([1], [17], [[0, -1]], INVALID), ([1, 0], [17, 16], [[0, 1], [9]], 0),
])
def test_tables(cas, q, kv, pages, code):
    prob = problem(cas, q, kv, pages=pages)
    n = ctypes.c_size_t(0)
    assert cas.load().cas_paged_chunk_workspace_size(ctypes.byref(prob.c), ctypes.byref(n)) == code


@pytest.mark.parametrize("field,value,code", [
    ("batch", 0, INVALID), ("group_size", 0, INVALID), ("head_dim", 96, UNSUPPORTED), ("page_size", 8, UNSUPPORTED),
    ("num_pages", 0, INVALID), ("kv_lens", None, INVALID), ("page_offsets", None, INVALID), ("num_kv_heads", 1 << 16, UNSUPPORTED),
    ("softmax_scale", 0.0, INVALID), ("softmax_scale", float("nan"), INVALID),
])
def test_problem_fields(cas, field, value, code):
    prob = problem(cas, [1], [4])
    setattr(prob.c, field, value)
    h, n = ctypes.c_void_p(), ctypes.c_size_t(0)
    assert cas.load().cas_paged_chunk_plan_create(ctypes.byref(prob.c), ctypes.byref(h), ctypes.byref(n)) == code and not h


@pytest.mark.parametrize("over,code", [
    (dict(q=None), INVALID), (dict(v=None), INVALID), (dict(o=None), INVALID), (dict(q=A + 8), ALIGN), (dict(lse=6 * A + 2), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(short=1), WORKSPACE), (dict(ws=5 * A + 8), ALIGN), (dict(o=A + 16), INVALID),
    (dict(o=2 * A), INVALID), (dict(lse=4 * A), INVALID), (dict(ws=3 * A), INVALID), (dict(ws=4 * A), INVALID),
])
def test_refusals(cas, over, code):
    prob = problem(cas, [40, 1], [3000, 7])
    a = dict(q=A, k=2 * A, v=3 * A, o=4 * A, ws=5 * A, lse=6 * A, short=0)
    a.update(over)
    n = cas.paged_chunk_workspace_size(prob) - a["short"]
    lib = cas.load()
    assert lib.cas_paged_chunk_fwd(ctypes.byref(prob.c), a["q"], a["k"], a["v"], a["o"], a["lse"], a["ws"], n, None) == code
    assert lib.cas_last_error_message()


def test_nothing_to_do(cas):
    prob = problem(cas, [0, 0], [5, 0])
    assert check(cas, [0, 0], [5, 0]).workgroups == 0
    assert cas.load().cas_paged_chunk_fwd(ctypes.byref(prob.c), None, None, None, None, None, None, 0, None) == 0


def test_plan_is_kept_while_the_tables_are(cas):
    prob = problem(cas, [1], [40])
    plan = prob.chunk_plan()
    assert prob.chunk_plan() is plan
    prob._kv[0] = 41
    assert prob.chunk_plan() is not plan


def test_binding_refusals(cas):
    import torch
    prob = problem(cas, [2, 1], [2, 17], pages=[[0], [1, 2]])
    bf = torch.bfloat16
    kp, q = torch.zeros(3, 16, 2, 64, dtype=bf), torch.zeros(3, 4, 64, dtype=bf)
    ok = dict(q=q, k_pages=kp, v_pages=kp.clone(), problem=prob)
    for over in (dict(q=q[:2]), dict(q=q[:, :3]), dict(q=torch.zeros(3, 4, 128, dtype=bf)[..., ::2]), dict(k_pages=kp[:2]),
                 dict(v_pages=kp.transpose(1, 2).contiguous().transpose(1, 2)), dict(o=q[:2]),
                 dict(lse=torch.zeros(4, 4)), dict(q=q[None]), {}):
        with pytest.raises(ValueError):                                    # ({}: not on a GPU)
            cas.paged_chunk_fwd(**{**ok, **over})
    for over in (dict(q=q.float()), dict(k_pages=kp.float()), dict(lse=torch.zeros(4, 3, dtype=bf))):
        with pytest.raises(TypeError):
            cas.paged_chunk_fwd(**{**ok, **over})


def test_few_whole_blocks_need_no_workspace(cas):
    """What fits the kernel's arguments: one block for a compute unit at most, and
    requests and granules within 960 words."""
    def needs(q, kv):
        own = [[100 * b + j for j in range(-(-L // 16))] for b, L in enumerate(kv)]
        return check(cas, q, kv, pages=own, Hkv=8, g=4, D=128).ws_bytes

    assert needs([33, 0, 5], [1100, 0, 70]) == needs([1] * 24, [300 + i for i in range(24)]) == 0
    assert needs([1] * 40, [300 + i for i in range(40)]) > 0      # 320 blocks
    assert needs([1] * 30, [600 + i for i in range(30)]) > 0      # 30 * (5 + 40) words
    assert needs([200], [9000]) > 0                               # cut
