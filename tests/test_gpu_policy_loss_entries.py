"""The clipped policy loss entry by entry: tolerances proportional to each entry of the gradient (policy_loss_bounds.py),
over the ranges of rows, actions, masks, strides and types."""
import numpy as np
import pytest
import torch

import policy_loss_ref as R
import test_gpu_policy_loss as L
from policy_loss_bounds import bounds

pytestmark = pytest.mark.gpu


def check(d):
    got = L.run(d)
    a = {k: L.to64(v) for k, v in dict(x=d["logits"], actions=d["actions"], old_logp=d["old_logp"], adv=d["advantages"], legal=d["legal"],
                                       weight=d["weight"], ref_logits=d["ref_logits"], ref_logp=d["ref_logp"]).items()}
    want = R.loss(**a, **L.COEF)
    tol = bounds(**a, **L.COEF, want=want, half_step=2.0 ** -8 if d["logits"].dtype is torch.bfloat16 else 2.0 ** -24)
    for n, ref, t in zip(("stats", "logp", "dlogits"), want, tol):
        have = L.to64(got[n])
        bad = ~(np.abs(have - ref) <= t)
        assert not bad.any(), (n, int(bad.sum()), np.argwhere(bad)[:4].tolist(), have[bad][:4], ref[bad][:4], t[bad][:4])


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("ref", ["logits", "logp", "none"])
@pytest.mark.parametrize("M,A", [(1, 1), (1, 6), (64, 6), (127, 5), (128, 8), (129, 17), (300, 20), (257, 21), (257, 32), (200, 33), (131, 64),
                                 (50, 65), (33, 127), (40, 1000), (9, 1024), (7, 1025), (5, 4099), (3, 8192), (3, 8200),
                                 (2, 20011), (3, 65536), (1, 300001)])
def test_entries(M, A, ref, dtype):
    check(L.make(M, A, dtype, ref, seed=M + A, weight=M % 2 == 1))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("spare", [0, 1, 2, 8])
@pytest.mark.parametrize("M,A", [(300, 6), (300, 20), (130, 64), (64, 100), (33, 512), (20, 1500), (3, 9001), (2, 65536)])
def test_entries_of_masked_and_strided_rows(M, A, spare, dtype):
    check(L.make(M, A, dtype, "logits", legal=True, spare=spare, seed=A, weight=True))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("M,A", [(50, 100), (20, 1500), (3, 9001)])
def test_a_reference_that_is_aligned_otherwise(M, A, dtype):
    """Logits that are slices of a wider output against dense rows."""
    d = L.make(M, A, dtype, "logits", spare=1, seed=A)
    d["ref_logits"] = d["ref_logits"].contiguous()
    check(d)


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("A", [6, 64, 100, 1500, 9001])
def test_entries_of_wide_distributions(A, dtype):
    """Logits of a spread of 40: most probabilities are 0 beside a few."""
    check(L.make(20, A, dtype, "logits", seed=A, scale=40.0))


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("M,A", [(607, 1500), (608, 1500), (608, 2048), (610, 2049), (608, 4096), (610, 4097), (2432, 4096), (2433, 1100)])
def test_rows_of_a_warp_or_a_cta(M, A, dtype):
    """Both sides of where a long row goes to a warp; some rows are compared."""
    d = L.make(M, A, dtype, "logits", legal=M % 2 == 0, seed=A, actions=torch.int64, weight=True)
    got = L.run(d)
    some = torch.tensor([0, 1, 303, M // 2, M - 9, M - 1], device="cuda")
    part = {k: v[some].contiguous() if isinstance(v, torch.Tensor) else v for k, v in d.items()}
    a = {k: L.to64(v) for k, v in dict(x=part["logits"], actions=part["actions"], old_logp=part["old_logp"], adv=part["advantages"],
                                       legal=part["legal"], weight=part["weight"], ref_logits=part["ref_logits"]).items()}
    want = R.loss(**a, **L.COEF)
    tol = bounds(**a, **L.COEF, want=want, half_step=2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24)
    for n, ref, t in zip(("logp", "dlogits"), want[1:], tol[1:]):
        assert (np.abs(L.to64(got[n][some]) - ref) <= t).all(), n
    assert abs(float(got["stats"][5]) - float(d["weight"].double()[got["logp"] != 0].sum())) <= 1e-6 * M


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("M,A", [(700, 65), (3000, 100), (700, 1501), (2500, 4096)])
def test_gradient_in_place_of_rows_of_a_warp(M, A, dtype):
    d = L.make(M, A, dtype, "logits", legal=True, seed=6)
    want = L.run(d)
    for _ in range(3):
        e = dict(d, logits=d["logits"].clone())
        got = L.run(e, dlogits=e["logits"])
        for n in ("stats", "logp", "dlogits"):
            assert torch.equal(got[n], want[n]), n
