"""How the chunk attention's launch tables reach the GPU, without a GPU: its host
code on stand-ins of the HIP runtime's entries (tests/table_slots_host.cpp). No
call waits for long, whatever becomes of the uploads before it."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("g++ not installed")
    exe = str(tmp_path_factory.mktemp("slots") / "table_slots_host")
    subprocess.run([cc, "-std=c++17", "-O1", "-rdynamic", "-pthread", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "table_slots_host.cpp"), "-o", exe, "-ldl"], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["usual", "never", "failing", "devices"])
def test_table_slots(program, scenario):
    from paper_2606_04557_amd import _lib
    r = subprocess.run([program, _lib.LIB_PATH, scenario], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
def test_calls_far_ahead_of_the_gpu(gpu_lib):
    """Forty calls behind 40 ms of other work on their stream: the tables of the
    later ones find no free slot and go as kernel arguments, with equal results."""
    import time
    import torch
    counts, kv = [300] * 24 + [1], [1000 + 13 * b for b in range(24)] + [77]
    pages, n = [], 0
    for L in kv:
        pages.append(list(range(n, n + -(-L // 16))))
        n += len(pages[-1])
    prob = gpu_lib.DecodeProblem(counts, kv, pages, n, 16, 2, 4, 128, 0.09)
    assert gpu_lib.paged_chunk_workspace_size(prob) > 0
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    q, kp, vp = rand(sum(counts), 8, 128), rand(n, 16, 2, 128), rand(n, 16, 2, 128)
    o, lse = gpu_lib.paged_chunk_fwd(q, kp, vp, prob)
    torch.cuda.synchronize()
    outs = [(torch.empty_like(o), torch.empty_like(lse)) for _ in range(40)]
    torch.cuda._sleep(80_000_000)   # cycles of at most 2.4 GHz
    t0 = time.perf_counter()
    for a, b in outs:
        gpu_lib.paged_chunk_fwd(q, kp, vp, prob, o=a, lse=b)
    assert time.perf_counter() - t0 > 0.01   # (some waited for a slot)
    torch.cuda.synchronize()
    assert all(torch.equal(a, o) and torch.equal(b, lse) for a, b in outs)
