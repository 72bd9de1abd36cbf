"""The bound on the error of beam selection's sums (csrc/cas_beam_error.h) against
the scan's arithmetic, step by step in numpy, without a GPU. The exponential is off
by its unit, upwards or downwards, as the instruction may be."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F, D = np.float32, np.float64
LOG2E = F(1.4426950408889634)
LN2 = 0.6931471805599453
J = 8


@pytest.fixture(scope="module")
def sum_error(tmp_path_factory):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("g++ not installed")
    at = tmp_path_factory.mktemp("sums")
    (at / "e.cpp").write_text('#include "cas_beam_error.h"\nextern "C" double f(double v, double s, double l, double m) { return cas::sum_error(v, s, l, m); }\n')
    lib = str(at / "e.so")
    subprocess.run([cc, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2606_04557_amd", "csrc"),
                    str(at / "e.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).f
    f.restype, f.argtypes = ctypes.c_double, [ctypes.c_double] * 4
    return f


def base_of(ref):
    return float(ref) if abs(ref) > 64 else float(F(ref * LOG2E)) * LN2


def scan(x, n, per_wave, unit):
    """[(sum, ref, low)] of a row's waves; n elements to a 16-byte piece, unit: what an exponential is multiplied with."""
    chunk = 64 * J * n
    x = np.concatenate([x, np.full(-len(x) % chunk, -np.inf, F)]).reshape(-1, J, 64, n)
    out = []
    for w in range(0, len(x), per_wave):
        ref = low = F(0)
        total, fresh = np.zeros(64), True
        for v in x[w: w + per_wave]:
            m = v[0].max(-1)
            while True:
                if fresh:
                    was, ref = base_of(ref), max(m.max(), np.finfo(F).min)
                    total = total * np.exp(was - base_of(ref)) if total.any() else total
                    if not (total > 1e-12).any():
                        low = ref
                with np.errstate(over="ignore", invalid="ignore"):
                    if abs(ref) <= 64:
                        t = (v.astype(D) * D(LOG2E) - D(F(ref * LOG2E))).astype(F)   # (one rounding)
                    else:
                        t = (v - ref) * LOG2E
                    e = (np.exp2(t.astype(D)) * unit).astype(F)
                h = n // 2
                while h:
                    e = e[..., :h] + e[..., h:2 * h]
                    h //= 2
                parts = np.zeros((2, 64), F)
                for j in range(J):
                    parts[j % 2] += e[j, :, 0]
                m = v.max((0, 2))
                fresh = bool((m - ref > 16).any())
                if not fresh:
                    break
            total = total + (parts[0] + parts[1]).astype(D)
        out.append((total.sum(), ref, low))
    return out


def check(sum_error, x, n, per_wave):
    """What the waves' sums come to, off by no more than sum_error says; returns the largest share of it that is used."""
    x = x.astype(F)
    most = float(x.max())
    exact = np.log(np.exp(x.astype(np.longdouble) - most).sum())
    share = 0.0
    for unit in (1 - 2.0 ** -23, 1.0, 1 + 2.0 ** -23):
        waves = scan(x, n, per_wave, unit)
        with np.errstate(under="ignore"):
            ln = max(np.log(sum(s * np.exp(base_of(r) - most) for s, r, _ in waves if s > 0)), 0.0)
        lowest = min(float(low) for s, r, low in waves if s > 0 and most - float(r) < 60)
        bound = sum_error(np.log(len(x)), ln, lowest, most)
        share = max(share, abs(float(ln - exact)) / bound)
        assert abs(ln - exact) <= bound <= 6e-6, (most, lowest, float(ln - exact), bound)
    return share


BAND = [0.0, 1.0, 30.0, 62.5, 63.0, 63.5, 64.0, 64.5, 65.0, 79.0, 81.0, 500.0, 1e4, 1e9, 1e18, 3e38]


@pytest.mark.parametrize("n", [8, 4])
@pytest.mark.parametrize("V", [1, 7, 2048, 32000])
def test_constant_rows(sum_error, n, V):
    """The least entropy to spare: all that is off is log2 e's rounding and the exponential's unit."""
    for c in BAND:
        for sign in (-1, 1):
            check(sum_error, np.full(V, sign * c), n, 1)


@pytest.mark.parametrize("n", [8, 4])
@pytest.mark.parametrize("std", [0.01, 1.0, 5.0])
def test_rows_around_the_border(sum_error, n, std):
    r = np.random.default_rng(int(100 * std) + n)
    for c in BAND[:12]:
        for sign in (-1, 1):
            for per_wave in (1, 4):
                check(sum_error, sign * c + std * r.standard_normal(20011), n, per_wave)


@pytest.mark.parametrize("n", [8, 4])
@pytest.mark.parametrize("rise", [1.0, 15.5, 16.5, 40.0])
def test_rows_that_rise_over_the_border(sum_error, n, rise):
    """A wave's first chunks below the border and the later ones above, and waves on both sides of it."""
    chunk = 64 * J * n
    for border in (-64.0, 64.0):
        for start in (-rise - 0.5, -rise / 2, -0.25, 0.25):
            for per_wave in (1, 2, 4):
                x = np.full(4 * chunk, border + start)
                x[chunk // 2:] += rise / 2
                x[chunk:] += rise / 2
                x[3 * chunk:] += rise
                check(sum_error, x, n, per_wave)
                check(sum_error, x[::-1].copy(), n, per_wave)
