"""Angles of far positions (cas_rope) against 80-bit arithmetic on the same
frequencies."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lo,hi", [(0, 1 << 12), (1 << 20, 1 << 21), ((1 << 31) - (1 << 20), (1 << 31) - 1)])
def test_angles(gpu_lib, lo, hi):
    """Pairs (1, 0) become (cos, sin): the reduced angle's rounding to fp32 is 2^-25
    (it is at most pi/4), the series and its roundings 1e-7, the result's 2^-25. (A
    rounded product of position and frequency would be off by up to 1.87e-7 radians
    more at the ends of int32, where the fastest pair is at 2^28 to 2^29 turns.)"""
    import torch
    T, D, R = 4096, 64, 64
    r = np.random.default_rng(lo)
    pos = (r.integers(lo, hi, T) * r.choice([-1, 1], T)).astype(np.int32)
    rope = gpu_lib.Rope(R, 1e4)
    x = torch.zeros((T, 1, D), device="cuda")
    x[..., : R // 2] = 1.0
    y, = gpu_lib.rope_fwd([x], torch.from_numpy(pos).cuda(), rope)
    a = oracle.rope.angles(pos, rope.turns)
    y = y.double().cpu().numpy()[:, 0]
    bar = 2.0 ** -25 + 1e-7 + 2.0 ** -25
    assert np.abs(y[:, : R // 2] - np.cos(a)).max() <= bar and np.abs(y[:, R // 2:] - np.sin(a)).max() <= bar
