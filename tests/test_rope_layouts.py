"""Rotary positions on tensors whose heads interleave in memory: slices of one
projection's output [tokens, heads, 3, d], which share a range of addresses and
no element. Tolerances are those of the equal bits: the rotation of an element
does not depend on where it lies."""
import ctypes

import pytest

INVALID = 1
A = 1 << 40   # addresses that are never touched


def call(heads_apart, tensors, tokens=10, D=64):
    import paper_2606_04557_amd as cas
    from paper_2606_04557_amd import _lib as L
    r = L.Rope(0, 64, A + (1 << 20), 1.0)
    ts = (L.RopeTensor * len(tensors))(*[
        L.RopeTensor(x=x, y=y, x_stride_tok=4 * heads_apart, x_stride_head=heads_apart, y_stride_tok=4 * heads_apart,
                     y_stride_head=heads_apart, heads=4) for x, y in tensors])
    return cas.load().cas_rope(ctypes.byref(r), 0, D, tokens, A, ts, len(tensors), 0, None)


@pytest.mark.parametrize("heads_apart,at", [
    (3 * 64, 0), (3 * 64, 32), (3 * 64, 3 * 64 - 32), (3 * 64, 3 * 64), (3 * 64, 9 * 64),   # heads overlap in part, or are the same
    (64 + 32, 64), (2 * 64, 64 + 8),                                                          # too little room beside a head
])
def test_heads_that_overlap_are_refused(heads_apart, at):
    x, z = 2 * A, 2 * A + 2 * at
    assert call(heads_apart, [(x, x), (z, 5 * A)]) == INVALID                 # an output over another input
    assert call(heads_apart, [(4 * A, x), (6 * A, z)]) == INVALID             # over another output


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("H,D", [(4, 64), (3, 128)])
def test_interleaved_heads(gpu_lib, T, H, D):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T + H)
    x = torch.randn((T, H, 3, D), generator=gen, device="cuda").to(torch.bfloat16)
    pos = torch.arange(100, 100 + T, dtype=torch.int32, device="cuda")
    rope = gpu_lib.Rope(D, 1e4)
    q, k, v = x[:, :, 0], x[:, :, 1], x[:, :, 2]
    want = [y.clone() for y in gpu_lib.rope_fwd([q.contiguous(), k.contiguous()], pos, rope)]
    # from the slices, and into slices of a buffer that is laid out like them
    assert all(torch.equal(a, b) for a, b in zip(gpu_lib.rope_fwd([q, k], pos, rope), want))
    y = torch.full_like(x, 7.0)
    gpu_lib.rope_fwd([q, k], pos, rope, outs=[y[:, :, 2], y[:, :, 0]])
    assert torch.equal(y[:, :, 2], want[0]) and torch.equal(y[:, :, 0], want[1]) and (y[:, :, 1] == 7.0).all()
    # in place; the values beside them stay
    kept = v.clone()
    gpu_lib.rope_fwd([q, k], pos, rope, outs=[q, k])
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, kept)
