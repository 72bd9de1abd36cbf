"""GPU parity of the copies between pages: every byte of the pools against copies made one by one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _t():
    import torch
    return torch


def make(n_pools, num_pages, page, shape, dtype, seed):
    t = _t()
    size = t.empty((), dtype=dtype).element_size()
    x = t.randint(0, 120, (n_pools, num_pages, page, *shape[:-1], shape[-1] * size), dtype=t.uint8,
                  generator=t.Generator().manual_seed(seed))
    return x.view(dtype)


def random_copies(num_pages, page, n, seed, whole=False, fan=True):
    r = np.random.default_rng(seed)
    ids = r.permutation(num_pages)
    dst, src = ids[:n], ids[n:]
    assert len(src) > 0
    s = r.choice(src, n) if fan else src[:n]
    rows = np.full(n, page) if whole else r.integers(0, page + 1, n)
    return np.stack([s, dst, rows], 1).astype(np.int32)


def expected(x, copies):
    y = x.clone()
    for s, d, n in np.asarray(copies).tolist():
        y[:, d, :n] = x[:, s, :n]
    return y


def same(a, b):
    t = _t()
    return t.equal(a.cpu().contiguous().view(t.uint8), b.contiguous().view(t.uint8))


@pytest.mark.parametrize("n_pools,num_pages,page,shape,dtype,n,whole", [
    (1, 2, 16, (8,), "bfloat16", 1, True), (2, 9, 16, (8, 128), "bfloat16", 4, False), (2, 700, 16, (8, 128), "bfloat16", 300, False),
    (2, 500, 16, (2, 64), "bfloat16", 240, True), (2, 500, 16, (2, 64), "bfloat16", 241, True), (64, 40, 16, (1, 64), "bfloat16", 20, False),
    (65, 40, 32, (1, 64), "uint8", 20, False), (130, 12, 16, (16,), "uint8", 3, False), (3, 50, 128, (3, 64), "float32", 24, False),
    (1, 5000, 16, (16,), "uint8", 2400, False), (4, 30, 64, (5, 48), "float16", 14, False), (1, 7, 128, (4, 4096), "float32", 3, False),
])
def test_copies(gpu_lib, n_pools, num_pages, page, shape, dtype, n, whole):
    t = _t()
    x = make(n_pools, num_pages, page, shape, getattr(t, dtype), n)
    copies = random_copies(num_pages, page, n, n_pools, whole)
    d = x.cuda()
    gpu_lib.pages_copy(list(d.unbind(0)), copies)
    ref = expected(x, copies)
    assert same(d, ref)
    pools = gpu_lib.PagePools(list(d.unbind(0)))
    gpu_lib.pages_copy(pools, copies)   # (again: the sources are as they were)
    gpu_lib.pages_copy(pools, copies[:0])
    assert same(d, ref)


def test_very_many_copies(gpu_lib):
    """More copies than one table has, 65,536, and pages of many pieces."""
    t = _t()
    n, num_pages = 150001, 310000
    x = t.randint(0, 120, (1, num_pages, 16, 16), dtype=t.uint8, generator=t.Generator().manual_seed(1))
    copies = random_copies(num_pages, 16, n, 2)
    d = x.cuda()
    gpu_lib.pages_copy([d[0]], copies)
    s, e, rows = (t.from_numpy(c).cuda().long() for c in copies.T)
    ref = x.cuda()
    ref[0, e] = t.where((t.arange(16, device="cuda") < rows[:, None])[..., None], ref[0, s], ref[0, e])
    assert t.equal(d, ref)
    assert int(d[0].long().sum()) != int(x[0].long().sum())


def test_copies_in_any_form(gpu_lib):
    """Lists, other integer types, a column-major array; another stream, the caller's workspace."""
    t = _t()
    x = make(2, 600, 16, (2, 64), t.bfloat16, 1)
    copies = random_copies(600, 16, 290, 3)
    ref = expected(x, copies)
    side = t.cuda.Stream()
    ws = t.empty(290 * 12 + 16, dtype=t.uint8, device="cuda")
    t.cuda.synchronize()
    for form, kw in ((copies.tolist(), {}), (copies.astype(np.int64), {}), (np.asfortranarray(copies), {}),
                     (copies, dict(stream=side)), (copies, dict(stream=side, workspace=ws))):
        d = x.cuda()
        side.wait_stream(t.cuda.current_stream())
        gpu_lib.pages_copy(list(d.unbind(0)), form, **kw)
        t.cuda.synchronize()
        assert same(d, ref)


def test_copy_binding_refusals(gpu_lib):
    t = _t()
    d = t.zeros((4, 10, 16, 32), dtype=t.bfloat16, device="cuda")
    for pools in ([d[0], d[1, :5]], [d[0], d[1].float()], [d[0].transpose(0, 1)], [d[0], d[1].cpu()], [d[0, :, 0, 0]]):
        with pytest.raises((ValueError, TypeError)):
            gpu_lib.PagePools(pools)
    for copies in ([[1, 2]], [1, 2, 3], [[1, 2, 17]], [[(1 << 32) + 1, 2, 1]], np.array([[1 << 40, 2, 1]]), [[1, 10, 1]], [[1, 2, 1], [3, 2, 1]], [[1, 2, 1], [2, 3, 1]]):
        with pytest.raises((ValueError, gpu_lib.CasError)):
            gpu_lib.pages_copy([d[0]], copies)
    with pytest.raises(TypeError):
        gpu_lib.pages_copy([d[0]], [[1.0, 2.0, 1.0]])
    with pytest.raises(gpu_lib.CasError):
        gpu_lib.pages_copy([d[0], d[0]], [[1, 2, 1]])
    with pytest.raises(gpu_lib.CasError):
        gpu_lib.pages_copy([d[0, :, :, :4].contiguous()], [[1, 2, 1]])   # (rows of 8 bytes)


def test_copies_past_four_gib(gpu_lib):
    t = _t()
    page = 128 * 4096
    d = t.zeros((9000, 128, 4096), dtype=t.uint8, device="cuda")   # 4.7 GB
    d[8999] = 3
    d[1] = 5
    gpu_lib.pages_copy([d], [[8999, 0, 128], [1, 8998, 77]])
    assert int(d[0].min()) == 3 and int(d[8998, :77].min()) == 5 and int(d[8998, 77:].max()) == 0 and int(d[8999].min()) == 3
    assert page == d[0].numel()


@pytest.mark.parametrize("n", [5, 300])
def test_copies_in_a_graph(gpu_lib, n):
    """A replay makes the copies that were captured, from what the pools hold then."""
    t = _t()
    x = make(2, 700, 16, (2, 64), t.uint8, n)
    copies = random_copies(700, 16, n, 1)
    d = x.cuda()
    pools = gpu_lib.PagePools(list(d.unbind(0)))
    ws = t.empty(12 * 300 + 16, dtype=t.uint8, device="cuda")
    passing = copies.copy()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        gpu_lib.pages_copy(pools, passing, workspace=ws)
    passing[:] = 0   # (read during the call)
    for i in range(4):
        x = make(2, 700, 16, (2, 64), t.uint8, 100 + i)
        d.copy_(x)
        other = make(1, 700, 16, (2, 64), t.uint8, i).cuda()
        gpu_lib.pages_copy([other[0]], random_copies(700, 16, 280, i))
        graph.replay()
        t.cuda.synchronize()
        assert same(d, expected(x, copies))


def test_tables_and_copies_keep_the_keys(gpu_lib):
    """Random forks, extensions, reorderings and compactions on a table, with their copies on the GPU: every
    sequence reads the rows that were written to it."""
    t = _t()
    r = np.random.default_rng(7)
    page, n_pages, row = 16, 120, 32
    table = gpu_lib.PageTable(n_pages, page)
    pools = [t.zeros((n_pages, page, row), dtype=t.int32, device="cuda") for _ in range(4)]
    cache = gpu_lib.PagePools(pools)
    held, count = {}, 0
    for step in range(60):
        ids = list(held)
        op = r.integers(0, 5)
        if op == 0 or not ids:
            parts = [int(r.choice(ids))] if ids and r.random() < 0.7 else []
            q = table.add(parts)
            held[q] = list(held[parts[0]]) if parts else []
        elif op == 1:
            qs = [int(q) for q in r.choice(ids, min(len(ids), 4), replace=False)]
            parents = [int(p) for p in r.integers(0, len(qs), len(qs))]
            table.reorder(qs, parents)
            old = [held[q] for q in qs]
            for q, p in zip(qs, parents):
                held[q] = list(old[p])
        elif op == 2 and len(ids) > 3:
            table.free([ids[0]])
            del held[ids[0]]
            gpu_lib.pages_copy(cache, table.compact())
        else:
            qs = [int(q) for q in r.choice(ids, min(len(ids), 3), replace=False)]
            counts = [int(c) for c in r.integers(0, 21, len(qs))]
            try:
                gpu_lib.pages_copy(cache, table.extend(qs, counts))
            except gpu_lib.CasError:
                table.free(ids[: len(ids) // 2])
                for q in ids[: len(ids) // 2]:
                    del held[q]
                continue
            lens, offs, pages = table.lists(qs)
            for i, (q, c) in enumerate(zip(qs, counts)):
                for j in range(lens[i] - c, lens[i]):
                    count += 1
                    for n, p in enumerate(pools):
                        p[pages[offs[i] + j // page], j % page] = 10 * count + n
                    held[q].append(10 * count)
    assert any(len(v) > 16 for v in held.values())
    for q, want in held.items():
        _, offs, pages = table.lists([q])
        at = t.tensor(list(pages[:offs[1]]), dtype=t.int64, device="cuda")
        for n, p in enumerate(pools):
            got = p[at].reshape(-1, row)[: len(want)].cpu()
            assert t.equal(got, (t.tensor(want, dtype=t.int32) + n)[:, None].expand(-1, row)), q
