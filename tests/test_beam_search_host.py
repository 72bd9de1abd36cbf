"""The loop of a beam search without a GPU: the selection is the oracle's, states are
reordered by indexing, and copies of pages are recorded instead of made."""
import types

import numpy as np
import pytest
import torch

import oracle

PAGE = 16


@pytest.fixture
def made(monkeypatch):
    """The search's GPU calls on CPU tensors. What is in `fail` raises instead."""
    import paper_2606_04557_amd as cas
    import paper_2606_04557_amd.beam as beam
    m = types.SimpleNamespace(cas=cas, copies=[], fail=set())

    def fails(name):
        if name in m.fail:
            raise MemoryError(name)

    def select(logits, scores, k, finished=None, pad_token=0):
        fails("beam_select")
        s, p, v = oracle.beam.select(logits.double().numpy(), scores.double().numpy(), k,
                                     None if finished is None else finished.numpy(), pad_token)
        return torch.from_numpy(s).float(), torch.from_numpy(p).int(), torch.from_numpy(v).int()

    def reorder(xs, parents, outs):
        fails("beam_reorder")
        for x, y in zip(xs, outs):
            y.copy_(torch.from_numpy(oracle.beam.reorder(x.numpy(), parents.numpy())))

    def copy(pools, copies):
        fails("pages_copy")
        m.copies.append(copies.tolist())

    def failing(name):
        method = getattr(cas.PageTable, name)

        def call(*a):
            fails(name)
            return method(*a)
        monkeypatch.setattr(cas.PageTable, name, call)

    monkeypatch.setattr(beam, "beam_select", select)
    monkeypatch.setattr(beam, "beam_reorder", reorder)
    monkeypatch.setattr(beam, "pages_copy", copy)
    for name in ("reorder", "truncate", "extend"):
        failing(name)
    return m


def pools_of(num_pages, row_bytes=256):
    x = torch.zeros((num_pages, PAGE, row_bytes), dtype=torch.uint8)
    return types.SimpleNamespace(pools=[x], num_pages=num_pages, page_size=PAGE, row_bytes=row_bytes)


def logits_of(batch, beams, vocab, seed):
    return torch.randn((batch, beams, vocab), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("what", ["beam_reorder", "reorder", "truncate", "extend", "pages_copy"])
def test_a_step_that_fails_ends_the_search(made, what):
    """Whatever fails after the selection leaves histories, pages and copies that may not belong together."""
    table = made.cas.PageTable(100, PAGE)
    prompts = [table.add(tokens=20), table.add(tokens=33)]
    before = table.info()
    search = made.cas.BeamSearch(table, pools_of(100), prompts, 3, 0, 10)
    search.step(logits_of(2, 1, 50, 1))
    x = logits_of(2, 3, 50, 2)
    x[0, :, 0] = 30.0   # (a beam ends)
    made.fail.add(what)
    with pytest.raises(MemoryError):
        search.step(x)
    made.fail.clear()
    for call in (lambda: search.step(logits_of(2, 3, 50, 3)), lambda: search.problem(1, 1, 64, 0.125)):
        with pytest.raises(RuntimeError):
            call()
    tokens, scores = search.results()
    assert tokens.shape == (2, 3, search.steps) and scores.shape == (2, 3)
    search.close()
    assert table.info() == before


def test_a_selection_that_fails_can_be_made_again(made):
    """Nothing has changed by then."""
    results = []
    for fail in (False, True):
        table = made.cas.PageTable(100, PAGE)
        search = made.cas.BeamSearch(table, pools_of(100), [table.add(tokens=20)], 3, 0, 4)
        search.step(logits_of(1, 1, 50, 1))
        if fail:
            made.fail.add("beam_select")
            with pytest.raises(MemoryError):
                search.step(logits_of(1, 3, 50, 2))
            made.fail.clear()
        for i in range(3):
            search.step(logits_of(1, 3, 50, 2 + i))
        assert search.done
        results.append((search.results(), table.info()))
    (a, i), (b, j) = results
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and i == j


def test_pools_with_more_pages_than_the_table(made):
    """The problem is one on the pools, as the paged calls ask for."""
    for pages in (100, 150):
        table = made.cas.PageTable(100, PAGE)
        search = made.cas.BeamSearch(table, pools_of(pages), [table.add(tokens=20)], 3, 0, 4)
        search.step(logits_of(1, 1, 50, 1))
        p = search.problem(2, 4, 64, 0.125)
        lens, offsets, ids = table.lists(search.seqs)
        assert (p.c.num_pages, p.c.page_size, p.c.num_kv_heads, p.c.group_size, p.c.head_dim) == (pages, PAGE, 2, 4, 64)
        assert list(p._qo) == [0, 1, 2, 3] and list(p._kv) == lens[:] == [21] * 3 and list(p._po) == offsets[:] and list(p._ids) == ids[:]


@pytest.mark.parametrize("row_bytes", [8, 24, 250])
def test_pools_whose_rows_cannot_be_copied(made, row_bytes):
    table = made.cas.PageTable(100, PAGE)
    prompt = table.add(tokens=20)
    before = table.info()
    with pytest.raises(ValueError):
        made.cas.BeamSearch(table, pools_of(100, row_bytes), [prompt], 3, 0, 4)
    assert table.info() == before


def test_a_search_that_cannot_be_made_leaves_the_table_as_it_was(made, monkeypatch):
    """Memory for the histories, or for the last of the forks, is not there."""
    table = made.cas.PageTable(100, PAGE)
    prompts = [table.add(tokens=20), table.add(tokens=5)]
    before, add, full, left = table.info(), made.cas.PageTable.add, torch.full, []

    def no_memory(*a, **kw):
        raise MemoryError

    def few(self, parts=(), tokens=0):
        if not left:
            raise MemoryError
        left.pop()
        return add(self, parts, tokens)

    monkeypatch.setattr(torch, "full", no_memory)
    with pytest.raises(MemoryError):
        made.cas.BeamSearch(table, pools_of(100), prompts, 3, 0, 4)
    monkeypatch.setattr(torch, "full", full)
    assert table.info() == before
    monkeypatch.setattr(made.cas.PageTable, "add", few)
    for n in range(6):
        left[:] = [0] * n
        with pytest.raises(MemoryError):
            made.cas.BeamSearch(table, pools_of(100), prompts, 3, 0, 4)
        assert table.info() == before
    for n in range(3):
        left[:] = [0] * n
        with pytest.raises(MemoryError):
            table.fork(prompts[0], 3)
        assert table.info() == before
