"""An infinite element of k or v (of q or do) makes the state's entries of its row or column infinite, of the sign that the
formulas give, in passes of steps and of chunks, and not NaN."""
import numpy as np
import pytest
import torch

import test_gpu_linattn as L

pytestmark = pytest.mark.gpu


def same_kind(have, want):
    return np.array_equal(np.isnan(have), np.isnan(want)) and np.array_equal(np.isposinf(have), np.isposinf(want)) and \
        np.array_equal(np.isneginf(have), np.isneginf(want))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("resets", [0, 0.02])
@pytest.mark.parametrize("name", ["k", "v", "q", "do"])
@pytest.mark.parametrize("T,K,V", [(5, 64, 64), (40, 64, 64), (130, 64, 64), (130, 128, 72), (700, 64, 40)])
def test_states_are_infinite_where_the_formulas_say(T, K, V, name, resets, dtype):
    d = L.make(T, 2, 2, K, V, dtype, seed=81, resets=resets, decay=-0.01)
    for at in (T - 1, T // 2, 0):
        for sign in (1, -1):
            e = dict(d)
            e[name] = d[name].clone()
            e[name][at, 1, 0, 5] = sign * float("inf")
            got = L.run(e)
            with np.errstate(invalid="ignore"):
                ref = L.reference(e)
            for n in ("s_last", "ds0"):
                assert same_kind(L.to64(got[n]), ref[n]), (n, at, sign)
            for n in ("o", "dq", "dk", "dv"):
                assert np.array_equal(np.isfinite(L.to64(got[n])), np.isfinite(ref[n])), (n, at, sign)
