"""bf16 outputs of linear attention are rounded once, whichever form a pass takes.

Tolerance.  An output is the rounding, 2^-8 of itself at most, of a sum that is off by `delta`.  Of the sum of
magnitudes (the same formulas over |q|, |k|, ...), delta is at most: 2^-17 for each of the operands that passes of
chunks hold in parts (the decayed products of two steps, the state, the decayed rows that make it), and
(2 K + 3 T + 16) roundings of 2^-24 of sums in fp32.  An operand of one bf16 part, off by up to 2^-8, would show
wherever the terms of an output nearly cancel.
"""
import numpy as np
import pytest
import torch

import test_gpu_linattn as L

pytestmark = pytest.mark.gpu


def within(have, want, mag, K, T):
    delta = (3 * 2.0 ** -17 + (2 * K + 3 * T + 16) * 2.0 ** -24) * mag
    return np.abs(have - want) <= 2.0 ** -8 * (np.abs(want) + delta) + delta + 1e-30


@pytest.mark.parametrize("T,N,H,K,V", [(64, 4, 2, 64, 64), (100, 3, 2, 50, 33), (130, 3, 2, 128, 96), (200, 1, 1, 64, 64),
                                       (70, 2, 3, 24, 128), (128, 40, 8, 64, 64)])
@pytest.mark.parametrize("resets", [0.0, 0.05])
def test_outputs_are_rounded_once(T, N, H, K, V, resets):
    d = L.make(T, N, H, K, V, torch.bfloat16, seed=21, resets=resets, lengths=N > 3, decay=-0.02)
    got, ref, mag = L.run(d), L.reference(d), L.reference(d, f=np.abs)
    for n in ("o", "dq", "dk", "dv"):
        bad = ~within(L.to64(got[n]), ref[n], mag[n], max(K, V), T)
        assert not bad.any(), (n, int(bad.sum()), np.argwhere(bad)[:4].tolist())


def test_the_tolerance_tells_one_part_from_two():
    """Outputs whose state alone is taken as one bf16 part, which the rounding of the result hides on average, are out of
    the tolerance."""
    d = L.make(64, 2, 2, 64, 64, torch.bfloat16, seed=22, resets=0.0, decay=-0.02)
    ref, mag = L.reference(d, backward=False), L.reference(d, f=np.abs, backward=False)
    s0 = d["s0"].bfloat16().float()
    one_part = L.reference(dict(d, s0=s0), backward=False)["o"]
    rounded = torch.from_numpy(one_part).bfloat16().double().numpy()
    assert not within(rounded, ref["o"], mag["o"], 64, 64).all()
    assert within(torch.from_numpy(ref["o"]).bfloat16().double().numpy(), ref["o"], mag["o"], 64, 64).all()
