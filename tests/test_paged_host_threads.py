"""Calls of the binding from several host threads at once, without a GPU: the
library's launches are stood in for, and CPU tensors say that they are on GPU 0.

A plan or a table that one thread uses must live until its call has returned,
whatever the others put in its place meanwhile.
"""
import gc

import pytest

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    """A CPU tensor that says it is on GPU 0."""

    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


class Library:
    """The library with some of its entries replaced."""

    def __init__(self, lib, **entries):
        self._lib = lib
        self.__dict__.update(entries)

    def __getattr__(self, name):
        return getattr(self._lib, name)


@pytest.fixture
def cas(monkeypatch):
    import paper_2606_04557_amd as cas
    cas.load()

    def on_device(index, stream, call):
        status = call(0)
        assert status == 0, status
    monkeypatch.setattr(cas, "_on_device", on_device)
    return cas


def replace_entries(cas, monkeypatch, **entries):
    lib = Library(cas.load(), **entries)
    monkeypatch.setattr(cas, "load", lambda: lib)


@pytest.mark.parametrize("call", ["append", "chunk"])
def test_a_plan_outlives_the_call_that_runs_it(cas, monkeypatch, call):
    """Another thread, which found no plan either, puts its own in the place of
    the one that the library is working on."""
    run, destroy = f"cas_paged_{call}_run", f"cas_paged_{call}_plan_destroy"
    real, destroyed, alive = getattr(cas.load(), destroy), [], []
    problem = cas.DecodeProblem([2, 1], [18, 5], [[0, 1], [2]], 4, 16, 2, 2, 64, 0.125)

    def run_stub(handle, *_):
        setattr(problem, f"_{call}_plan", None)
        gc.collect()
        alive.append(handle.value not in destroyed)
        return 0

    def destroy_stub(handle):
        destroyed.append(handle.value)
        return real(handle)
    replace_entries(cas, monkeypatch, **{run: run_stub, destroy: destroy_stub})
    pools = on_gpu(4, 16, 2, 64), on_gpu(4, 16, 2, 64)
    if call == "append":
        cas.paged_append(on_gpu(3, 2, 64), on_gpu(3, 2, 64), *pools, problem)
    else:
        cas.paged_chunk_fwd(on_gpu(3, 4, 64), *pools, problem, o=on_gpu(3, 4, 64), lse=on_gpu(4, 3, dtype=torch.float32),
                            workspace=on_gpu(1 << 20, dtype=torch.uint8))
    gc.collect()
    assert alive == [True]
    assert len(destroyed) == 1   # (and it is freed afterwards)


def test_frequencies_outlive_every_call_that_reads_them(cas, monkeypatch):
    """Two threads whose first calls with one Rope come at the same time both
    upload its frequencies: each call has to get an upload that is kept."""
    import threading
    import weakref
    both, uploads, read = threading.Barrier(2, timeout=30), [], []

    class Stream:
        cuda_stream = 0

    def upload(*args, **kw):
        t = torch.zeros(32, dtype=torch.float64)
        uploads.append((t.data_ptr(), weakref.ref(t)))
        both.wait()          # (neither has stored its own yet)
        return t

    def rope_stub(c, *_):
        both.wait()          # (both have)
        gc.collect()
        read.append(any(ref() is not None and at == c.turns for at, ref in uploads))
        both.wait()
        return 0
    rope = cas.Rope(64)
    replace_entries(cas, monkeypatch, cas_rope=rope_stub)
    monkeypatch.setattr(torch, "tensor", upload)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: Stream)
    failed = []

    def work():
        try:
            x = on_gpu(4, 2, 64)
            cas.rope_fwd([x], on_gpu(4, dtype=torch.int32), rope, outs=[x])
        except BaseException as e:   # noqa: BLE001
            failed.append(e)
            both.abort()
    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    assert len(uploads) == 2 and read == [True, True]
    assert sum(ref() is not None for _, ref in uploads) == 1   # (one is kept)


@pytest.mark.gpu
def test_first_calls_of_threads_on_the_gpu(gpu_lib):
    """Four threads whose first calls on one problem and one Rope come together, each
    with its own stream and pools: the bits of calls one after the other."""
    import threading
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    counts, kv, pages, n = [], [], [], 0
    for b in range(30):
        counts.append(1 + b % 7)
        kv.append(counts[-1] + 61 * b)
        pages.append(list(range(n, n + -(-kv[-1] // 16))))
        n += len(pages[-1])
    T = sum(counts)
    x, base = rand(T, 12, 64), [rand(n, 16, 2, 64) for _ in range(2)]
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]

    def step(problem, rope, pools, stream):
        rotated = gpu_lib.paged_append(k, v, *pools, problem, rope=rope, q=q, stream=stream)
        return gpu_lib.paged_chunk_fwd(rotated, *pools, problem, stream=stream)
    make = lambda: (gpu_lib.DecodeProblem(counts, kv, pages, n, 16, 2, 4, 64, 0.125), gpu_lib.Rope(64, 1e4))
    pools = [[p.clone() for p in base] for _ in range(5)]
    want = step(*make(), pools[4], None)
    torch.cuda.synchronize()
    bad = []

    def work(i, problem, rope, start):
        try:
            s = torch.cuda.Stream()
            start.wait(30)
            got = step(problem, rope, pools[i], s)
            s.synchronize()
            if not all(torch.equal(a, b) for a, b in zip((*got, *pools[i]), (*want, *pools[4]))):
                bad.append(i)
        except BaseException as e:   # noqa: BLE001
            bad.append(e)
    for _ in range(10):
        start, shared = threading.Barrier(4), make()
        threads = [threading.Thread(target=work, args=(i, *shared, start)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not bad, bad
