"""The host-side tests of the rotary positions, of appending and of the chunk
attention (argument checks, plans) against a build with AddressSanitizer and
UndefinedBehaviorSanitizer on its host code. Needs hipcc, no GPU."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not installed")
def test_paged_host_code_under_asan_and_ubsan(tmp_path):
    hits = sorted(glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    if not hits:
        pytest.skip("clang AddressSanitizer runtime not found")
    from paper_2606_04557_amd import build
    sources = glob.glob(os.path.join(build.CSRC, "*")) + glob.glob(os.path.join(build.INCLUDE, "*")) + [build.__file__]
    lib = build.SAN_LIB_PATH
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(f) for f in sources):
        lib = build.build(sanitize=True)
    env = dict(os.environ)
    env["CAS_LIB"] = lib
    env["LD_PRELOAD"] = hits[-1] + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    log = str(tmp_path / "san")
    env["ASAN_OPTIONS"] = f"detect_leaks=0:abort_on_error=1:log_path={log}"
    env["UBSAN_OPTIONS"] = f"print_stacktrace=1:log_path={log}"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "tests/test_rope_append_host.py",
                        "tests/test_chunk_plan.py"], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True,
                       timeout=600)
    reports = "".join(open(f).read() for f in glob.glob(log + "*"))
    assert r.returncode == 0 and not reports, (r.stdout[-3000:], reports[:3000])
