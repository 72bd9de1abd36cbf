"""Page tables, copies of pages, beam selection and reordering without a GPU: the
oracle's pins, the page table against a model of it, and every refusal (argument
checks run before any HIP call, so made-up addresses stand in for device memory)."""
import ctypes
import random

import numpy as np
import pytest

import oracle

A = 1 << 40   # stands in for device memory


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
def test_oracle_select_pins():
    inf = np.inf
    # Probabilities 1/2, 1/4, 1/4 and 1/4, 1/4, 1/2.
    x = np.log([[[2.0, 1.0, 1.0], [1.0, 1.0, 2.0]]])
    s, p, t = oracle.beam.select(x, [[0.0, 0.0]], 6)
    assert np.allclose(np.exp(s[0]), [0.5, 0.5, 0.25, 0.25, 0.25, 0.25])
    assert p[0].tolist() == [0, 1, 0, 0, 1, 1] and t[0].tolist() == [0, 2, 1, 2, 0, 1]
    # A beam that has ended keeps its score; one that is out of the search has nothing; -inf ones follow in order.
    s, p, t = oracle.beam.select(x, [[-0.1, -inf]], 5, finished=[[True, False]], pad=2)
    assert s[0].tolist() == [-0.1] + [-inf] * 4 and (p[0] * 3 + t[0]).tolist() == [2, 0, 1, 3, 4]
    for bad in (np.nan, inf):
        y = x.copy()
        y[0, 0, 1] = bad
        s, p, t = oracle.beam.select(y, [[0.0, 0.0]], 3)
        assert p[0].tolist() == [1, 1, 1] and t[0].tolist() == [2, 0, 1]
    y = np.full((1, 1, 4), -3.4e38)
    s, p, t = oracle.beam.select(y, [[-2.0]], 4)
    assert np.allclose(s, -2.0 - np.log(4)) and t[0].tolist() == [0, 1, 2, 3]


def test_oracle_reorder_pins():
    x = np.arange(12).reshape(2, 3, 2)
    assert oracle.beam.reorder(x, [[2, 2], [0, 1]]).tolist() == [[[4, 5], [4, 5]], [[6, 7], [8, 9]]]


# -- the page table -----------------------------------------------------------
class Model:
    """What the sequences hold, token by token: every page's rows with what was written there."""

    def __init__(self, page):
        self.page, self.rows, self.seqs, self.n = page, {}, {}, 0

    def write(self, lists, seq, start, count):
        """The new tokens of a sequence go to their places, as paged_append has them."""
        for j in range(start, start + count):
            self.n += 1
            self.rows[(lists[j // self.page], j % self.page)] = self.n
            self.seqs[seq].append(self.n)

    def copy(self, copies):
        assert len({c[1] for c in copies}) == len(copies) and not {c[0] for c in copies} & {c[1] for c in copies}
        for s, d, n in copies:
            for r in range(n):
                self.rows[(d, r)] = self.rows.get((s, r))

    def check(self, table):
        ids = list(self.seqs)
        lens, offs, pages = table.lists(ids)
        used = set()
        for i, q in enumerate(ids):
            mine = pages[offs[i]:offs[i + 1]]
            assert lens[i] == len(self.seqs[q]) and len(mine) == -(-lens[i] // self.page)
            assert [self.rows[(mine[j // self.page], j % self.page)] for j in range(lens[i])] == self.seqs[q]
            used |= set(mine)
        info = table.info()
        assert info == dict(sequences=len(ids), pages_used=len(used), pages_free=table.num_pages - len(used),
                            pages_end=max(used) + 1 if used else 0)


@pytest.mark.parametrize("seed", range(12))
def test_page_table_keeps_what_sequences_hold(cas, seed):
    """Random calls on a table and on a model that writes every token to its place:
    every sequence reads its own tokens back, and no page is lost or given twice."""
    r = random.Random(seed)
    page, n_pages = r.choice([16, 32]), r.choice([40, 200])
    t, m = cas.PageTable(n_pages, page), Model(page)

    def tables(q):
        lens, offs, pages = t.lists([q])
        return list(pages[:offs[1]])

    for _ in range(150):
        op, ids = r.choice(["add", "add", "extend", "extend", "extend", "reorder", "truncate", "free", "compact"]), list(m.seqs)
        before = t.info()
        try:
            if op == "add":
                parts = [q for q in r.sample(ids, min(len(ids), r.randint(0, 3)))]
                parts = [q for q in parts[:-1] if len(m.seqs[q]) % page == 0] + parts[-1:]
                if r.random() < 0.3:
                    parts = [q for q in parts if len(m.seqs[q]) % page == 0] * 2
                if sum(len(m.seqs[q]) for q in parts) < 400:
                    q = t.add(parts)
                    m.seqs[q] = [x for p in parts for x in m.seqs[p]]
            elif op == "extend" and ids:
                qs = r.sample(ids, r.randint(1, len(ids)))
                counts = [r.choice([0, 1, 1, r.randint(0, 2 * page)]) for _ in qs]
                lens = [len(m.seqs[q]) for q in qs]
                m.copy(t.extend(qs, counts).tolist())
                for q, n, c in zip(qs, lens, counts):
                    m.write(tables(q), q, n, c)
            elif op == "reorder" and ids:
                qs = r.sample(ids, r.randint(1, len(ids)))
                parents = [r.randrange(len(qs)) for _ in qs]
                t.reorder(qs, parents)
                old = [list(m.seqs[q]) for q in qs]
                for q, p in zip(qs, parents):
                    m.seqs[q] = list(old[p])
            elif op == "truncate" and ids:
                q = r.choice(ids)
                n = r.randint(0, len(m.seqs[q]))
                t.truncate(q, n)
                del m.seqs[q][n:]
            elif op == "free" and ids and r.random() < 0.6:
                qs = r.sample(ids, r.randint(1, min(3, len(ids))))
                t.free(qs)
                for q in qs:
                    del m.seqs[q]
            elif op == "compact":
                most = r.choice([None, 0, 1, 3])
                moves = t.compact(most).tolist()
                m.copy(moves)
                assert all(d < s for s, d, _ in moves)
                if most is None:
                    assert t.info()["pages_end"] == t.info()["pages_used"]
        except cas.CasError as e:
            assert e.status == 8 and op == "extend" and t.info() == before   # CAS_ERR_PAGES, and nothing changed
        m.check(t)
    t.free(list(m.seqs))
    assert t.info() == dict(sequences=0, pages_used=0, pages_free=n_pages, pages_end=0)


def test_extend_leaves_the_last_owner_its_page(cas):
    t = cas.PageTable(10, 16)
    q = t.add(tokens=20)
    a, b = t.fork(q, 2)
    assert t.extend([q, a, b], [1, 0, 1]).tolist() == [[1, 2, 4], [1, 3, 4]]   # a's, which is not extended
    assert t.extend([a], [1]).tolist() == []
    assert t.extend([a, b], [0, 0]).tolist() == []
    # a page twice in one sequence: its second place is only partly in use
    c = t.add(tokens=16)
    d = t.add([c, c])
    t.free([c])
    t.truncate(d, 20)
    assert t.extend([d], [1]).tolist() == [[4, 5, 4]]
    assert t.lists([d])[2][:] == [4, 5]


def test_page_table_refusals(cas, L):
    bad, few = L.CAS_ERR_INVALID_ARGUMENT, L.CAS_ERR_PAGES

    def refused(code, call):
        with pytest.raises(cas.CasError) as e:
            call()
        assert e.value.status == code, e.value

    for n, p, code in ((0, 16, bad), (1 << 31, 16, bad), (4, 17, L.CAS_ERR_UNSUPPORTED), (4, 0, L.CAS_ERR_UNSUPPORTED)):
        refused(code, lambda: cas.PageTable(n, p))
    t = cas.PageTable(4, 16)
    q = t.add(tokens=20)
    gone = t.add()
    t.free([gone])
    for call in (lambda: t.add([gone]), lambda: t.add([q, q]), lambda: t.extend([gone], [1]), lambda: t.extend([q, q], [1, 1]),
                 lambda: t.extend([q], [-1]), lambda: t.reorder([q], [1]), lambda: t.reorder([q], [-1]), lambda: t.reorder([q, q], [0, 0]),
                 lambda: t.truncate(q, 21), lambda: t.truncate(q, -1), lambda: t.truncate(gone, 0), lambda: t.free([gone]),
                 lambda: t.free([q, q]), lambda: t.lists([gone])):
        before = t.info(), t.lists([q])[2][:]
        refused(bad, call)
        assert (t.info(), t.lists([q])[2][:]) == before
    refused(few, lambda: t.extend([q], [45]))
    refused(L.CAS_ERR_UNSUPPORTED, lambda: t.extend([q], [1 << 30]))
    for call in (lambda: t.extend([q], [1, 2]), lambda: t.reorder([q], [0, 0]), lambda: t.compact(-1), lambda: t.add([q], tokens=1)):
        with pytest.raises(ValueError):
            call()
    assert t.info()["sequences"] == 1 and t.extend([q], [44]).tolist() == []
    lib, n, seq = cas.load(), ctypes.c_int32(), ctypes.c_int64()
    one, ids = (ctypes.c_int64 * 1)(q), (ctypes.c_int32 * 9)()
    assert lib.cas_page_table_create(4, 16, None) == bad
    assert lib.cas_page_table_info(None, ctypes.byref(L.PageTableInfo())) == bad and lib.cas_page_table_info(t.h, None) == bad
    assert lib.cas_page_table_add(t.h, None, 1, ctypes.byref(seq)) == bad and lib.cas_page_table_add(t.h, one, -1, ctypes.byref(seq)) == bad
    assert lib.cas_page_table_add(t.h, one, 1, None) == bad and lib.cas_page_table_add(None, one, 1, ctypes.byref(seq)) == bad
    assert lib.cas_page_table_extend(t.h, one, 1, ids, None, ctypes.byref(n)) == bad
    assert lib.cas_page_table_extend(t.h, one, 1, None, ids, ctypes.byref(n)) == bad
    assert lib.cas_page_table_extend(t.h, one, 1, ids, ids, None) == bad
    assert lib.cas_page_table_reorder(t.h, one, 1, None) == bad and lib.cas_page_table_reorder(None, one, 1, ids) == bad
    assert lib.cas_page_table_free(None, one, 1) == bad and lib.cas_page_table_truncate(None, 0, 0) == bad
    assert lib.cas_page_table_compact(t.h, 1, None, ctypes.byref(n)) == bad
    assert lib.cas_page_table_lists(t.h, one, 1, ids, None, ids, 9) == bad
    assert lib.cas_page_table_lists(t.h, one, 1, None, ids, ids, 9) == bad
    assert lib.cas_page_table_lists(t.h, one, 1, ids, (ctypes.c_int32 * 2)(), ids, 3) == bad   # (of four)
    assert lib.cas_page_table_destroy(None) == 0


def test_problem_of_a_table(cas):
    t = cas.PageTable(64, 16)
    c = [t.add(tokens=32), t.add(tokens=48)]
    q = [t.add([c[1], c[0]]), t.add([c[0]])]
    t.extend(q, [5, 17])
    p = t.problem(q, [2, 17], 2, 4, 64, 0.125)
    assert list(p._qo) == [0, 2, 19] and list(p._kv) == [85, 49] and list(p._po) == [0, 6, 10] and p.Tq == 19
    assert list(p._ids[:10]) == [2, 3, 4, 0, 1, 5, 0, 1, 6, 7]
    assert cas.paged_chunk_workspace_size(p) >= 0   # (planned: the tables are in order)
    with pytest.raises(ValueError):
        t.problem(q, [1], 2, 4, 64, 0.125)


def test_problem_of_tables_that_do_not_fit(cas):
    """Arrays shorter than what the library would read of them, or of another type, are refused."""
    t = cas.PageTable(64, 16)
    q = [t.add(tokens=40), t.add(tokens=20)]
    lens, offs, ids = t.lists(q)
    ints = lambda *v: (ctypes.c_int32 * len(v))(*v)
    rest = (64, 16, 2, 4, 64, 0.125)
    assert cas.DecodeProblem.from_tables([1, 1], lens, offs, ids, *rest).Tq == 2
    for counts, tables in (([1, 1], (ints(40), offs, ids)), ([1, 1], (lens, offs, ints(*ids[:4]))), ([1, 1], (lens, ints(0, 3), ids)),
                           ([1], (lens, offs, ids)), ([1, 1], (lens, ints(0, 3, 1 << 30), ids))):
        with pytest.raises(ValueError):
            cas.DecodeProblem.from_tables(counts, *tables, *rest)
    for tables in (((ctypes.c_int64 * 2)(40, 20), offs, ids), (lens, list(offs), ids), (lens, offs, np.array(ids[:], dtype=np.int32))):
        with pytest.raises(TypeError):
            cas.DecodeProblem.from_tables([1, 1], *tables, *rest)


# -- copies of pages ----------------------------------------------------------
def _copy(cas, copies, pools=(A, A + (1 << 30)), num_pages=100, page=16, row=256, ws=0, ws_bytes=0, n=None, at=True):
    a = (ctypes.c_int32 * (3 * max(len(copies), 1)))(*[x for c in copies for x in c])
    p = (ctypes.c_void_p * max(len(pools), 1))(*pools)
    return cas.load().cas_pages_copy(p if at else None, len(pools), num_pages, page, row, ctypes.addressof(a),
                                     len(copies) if n is None else n, ws, ws_bytes, None)


def test_copy_refusals(cas, L):
    bad, unsupported, align = L.CAS_ERR_INVALID_ARGUMENT, L.CAS_ERR_UNSUPPORTED, L.CAS_ERR_ALIGNMENT
    ok = [(1, 2, 16)]
    for kw, code in ((dict(page=17), unsupported), (dict(num_pages=0), bad), (dict(num_pages=1 << 31), bad), (dict(row=0), bad),
                     (dict(row=24), align), (dict(row=1 << 25), unsupported), (dict(n=-1), bad), (dict(at=False), bad),
                     (dict(pools=(A, 0)), bad), (dict(pools=(A, A + 8)), align), (dict(pools=(A, A)), bad),
                     (dict(pools=(A, A + 100 * 16 * 256 - 16)), bad), (dict(pools=(A, A + (1 << 30), A)), bad)):
        assert _copy(cas, ok, **kw) == code, kw
    for copies in ([(1, 100, 1)], [(100, 1, 1)], [(-1, 1, 1)], [(1, -1, 1)], [(1, 2, 17)], [(1, 2, -1)], [(1, 1, 3)], [(1, 2, 3), (3, 2, 3)],
                   [(1, 2, 3), (2, 4, 3)], [(1, 2, 3), (5, 6, 0), (6, 4, 3)]):
        assert _copy(cas, copies) == bad, copies
    assert _copy(cas, []) == 0 and _copy(cas, [(1, 2, 0)]) == 0 and _copy(cas, ok, pools=()) == 0
    # long lists need a workspace
    many, size = [(i, 1000 + i, 16) for i in range(241)], ctypes.c_size_t()
    lib = cas.load()
    for n, want in ((0, 0), (240, 0), (241, 2896)):
        assert lib.cas_pages_copy_workspace_size(n, ctypes.byref(size)) == 0 and size.value == want
    assert lib.cas_pages_copy_workspace_size(-1, ctypes.byref(size)) == bad and lib.cas_pages_copy_workspace_size(1, None) == bad
    assert _copy(cas, many, num_pages=2000) == L.CAS_ERR_WORKSPACE and lib.cas_last_workspace_needed() == 2896
    assert _copy(cas, many, num_pages=2000, ws=A - 4096, ws_bytes=2895) == L.CAS_ERR_WORKSPACE
    assert _copy(cas, many, num_pages=2000, ws=A - 4096 + 8, ws_bytes=2896) == align
    assert _copy(cas, many, num_pages=2000, ws=A + 4096, ws_bytes=2896) == bad   # inside a pool


def test_copy_binding_refusals(cas):
    import torch
    with pytest.raises(ValueError):
        cas.PagePools([])
    with pytest.raises(ValueError):
        cas.PagePools([torch.zeros(4, 16, 2)])   # (not on a GPU)


# -- beam selection -----------------------------------------------------------
def _beam(cas, L, fields=(), logits=A, scores=A + (1 << 34), finished=0, outs=(A + (2 << 34), A + (3 << 34), A + (4 << 34)),
          ws=A + (5 << 34), ws_bytes=1 << 30):
    p = L.BeamProblem(L.CAS_DTYPE_BF16, 2, 4, 8, 1000, 1000, 0)
    for f, v in dict(fields).items():
        setattr(p, f, v)
    size = ctypes.c_size_t(77)
    code = cas.load().cas_beam_select_workspace_size(ctypes.addressof(p), ctypes.byref(size))
    return code, size.value, cas.load().cas_beam_select(ctypes.addressof(p), logits, scores, finished, *outs, ws, ws_bytes, None)


def test_beam_refusals(cas, L):
    bad, unsupported, align = L.CAS_ERR_INVALID_ARGUMENT, L.CAS_ERR_UNSUPPORTED, L.CAS_ERR_ALIGNMENT
    for f, v, code in (("dtype", 2, unsupported), ("batch", -1, bad), ("beams", 0, bad), ("beams", 65, unsupported), ("k", 0, bad),
                       ("k", 65, unsupported), ("vocab", 0, bad), ("vocab", 1, bad), ("vocab", (1 << 30) + 1, unsupported),
                       ("row_stride", 999, bad), ("row_stride", 1 << 41, bad), ("pad_token", -1, bad), ("pad_token", 1000, bad),
                       ("batch", (1 << 18) + 1, unsupported)):
        size, _, call = _beam(cas, L, {f: v})
        assert size == code and call == code, (f, v)
    assert _beam(cas, L, {"batch": 0}) == (0, 0, 0)
    for kw, code in ((dict(logits=0), bad), (dict(scores=0), bad), (dict(outs=(0, A + 64, A + 128)), bad), (dict(logits=A + 1), align),
                     (dict(scores=A + (1 << 34) + 2), align), (dict(outs=(A + 2, A + 64, A + 128)), align),
                     (dict(scores=A + 64), 0), (dict(outs=(A + 64, A + (3 << 34), A + (4 << 34))), bad),
                     (dict(outs=(A + (2 << 34), A + (2 << 34) + 60, A + (4 << 34))), bad), (dict(ws=A + 4096), bad),
                     (dict(ws=0), L.CAS_ERR_WORKSPACE), (dict(ws_bytes=100), L.CAS_ERR_WORKSPACE), (dict(ws=A + (5 << 34) + 8), align),
                     (dict(finished=A + (2 << 34)), bad)):
        if code:
            assert _beam(cas, L, **kw)[2] == code, kw
    assert cas.load().cas_beam_select_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == bad
    assert cas.load().cas_beam_select_workspace_size(ctypes.addressof(L.BeamProblem()), None) == bad


def test_beam_binding_refusals(cas):
    import torch
    x, s = torch.zeros(2, 4, 100), torch.zeros(2, 4)
    for logits in (x[0], x.transpose(0, 1)[:, :1].expand(4, 2, 100).transpose(1, 2), x.expand(3, 2, 4, 100)[:, 0, :2].transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            cas.beam_select(logits, s)
    for args in ((x, s), (x, s[:1]), (x, s.double()), (x.half(), s), (x, torch.zeros(4, 2).t())):
        with pytest.raises((ValueError, TypeError)):
            cas.beam_select(*args)   # (the first: not on a GPU)
    for outs in (None, [x, x]):
        with pytest.raises((ValueError, TypeError)):
            cas.beam_reorder([x], torch.zeros(2, 4, dtype=torch.int32), outs=outs)


# -- reordering ---------------------------------------------------------------
def _reorder(cas, L, *states, parents=A + (9 << 34), batch=2, beams_in=4, beams_out=4, n=None):
    a = (L.BeamState * max(len(states), 1))(*[L.BeamState(*s) for s in states])
    return cas.load().cas_beam_reorder(parents, batch, beams_in, beams_out, ctypes.addressof(a), len(states) if n is None else n, None)


def test_reorder_refusals(cas, L):
    bad, unsupported = L.CAS_ERR_INVALID_ARGUMENT, L.CAS_ERR_UNSUPPORTED
    B = A + (1 << 34)
    ok = (A, B, 100, 512, 128, 512, 128)
    for kw, code in ((dict(batch=-1), bad), (dict(beams_in=0), bad), (dict(beams_out=0), bad), (dict(beams_in=65), unsupported),
                     (dict(beams_out=65), unsupported), (dict(parents=0), bad), (dict(parents=A + (9 << 34) + 2), L.CAS_ERR_ALIGNMENT),
                     (dict(n=0), bad), (dict(n=9), bad), (dict(batch=1 << 19), unsupported), (dict(parents=B), bad)):
        assert _reorder(cas, L, ok, **kw) == code, kw
    for s in ((0, B, 100, 512, 128, 512, 128), (A, 0, 100, 512, 128, 512, 128), (A, B, -1, 512, 128, 512, 128), (A, B, 100, -1, 128, 512, 128),
              (A, B, 100, 512, 128, 512, 99), (A, B, 100, 512, 128, 483, 128), (A, A + 512, 100, 512, 128, 512, 128),
              (A, A, 100, 512, 128, 1024, 128), (A, A, 100, 512, 128, 512, 256), (A, B, 100, 512, 128, 512, 0), (A, B, 100, 512, 128, 0, 128)):
        assert _reorder(cas, L, s) == bad, s
    assert _reorder(cas, L, (A, A, 100, 512, 128, 512, 128), beams_out=3) == bad
    assert _reorder(cas, L, ok, (B, A, 100, 512, 128, 512, 128)) == bad        # each other's x
    assert _reorder(cas, L, ok, (A + 4096, B + 64, 100, 512, 128, 512, 128)) == bad
    assert _reorder(cas, L, ok, batch=0) == 0 and _reorder(cas, L, (0, 0, 0, 0, 0, 0, 0)) == 0
