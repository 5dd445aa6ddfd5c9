"""Linear attention whose states come near the largest fp32 number: what the formulas keep finite is finite.
The reference and the tolerances are those of test_gpu_linattn.py."""
import pytest
import torch

import test_gpu_linattn as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("large", ["v", "do"])
@pytest.mark.parametrize("decay", [0.0, -0.05, -0.5, -0.69, -1.0, -2.0, -3.0, -40.0])
@pytest.mark.parametrize("T,K,V", [(2, 64, 64), (9, 64, 64), (9, 16, 20), (19, 32, 40), (40, 64, 64), (33, 128, 128), (300, 40, 72)])
def test_large_states(T, K, V, decay, large, dtype):
    """The forward state (large v) or the gradient's (large do) is a sum of terms of 4e36 / (1 - g) and more; it leaves the
    range if it is kept times 2^7 or more.  The other operands are small, so that every result stays within."""
    d = L.make(T, 2, 2, K, V, dtype, seed=31, decay=decay, resets=0.2)
    big = 2.0 ** 121 * (1 - torch.exp(torch.tensor(decay)).item() * 0.98)
    small = 2.0 ** -10
    for n in ("q", "k", "v", "do"):
        d[n] = (d[n].float().clamp(-4, 4) * (big / 8 if n == large else 1.0 if n == dict(v="k", do="q")[large] else small)).to(dtype)
    d["s0"] *= 2.0 ** 122 if large == "v" else small
    d["ds_last"] *= 2.0 ** 122 if large == "do" else small
    got = L.check(d)
    assert all(torch.isfinite(t.float()).all() for t in got.values())


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("decay", [-0.05, -0.69, -2.0, -40.0])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17])
def test_ends_of_windows(T, decay, dtype):
    """Passes that end within, at and behind a window, in either direction, with a reset at the first and the last step."""
    d = L.make(T, 3, 2, 48, 40, dtype, seed=32 + T, decay=decay, resets=0.1)
    d["reset"][0, 1] = d["reset"][T - 1, 2] = 1
    L.check(d)
