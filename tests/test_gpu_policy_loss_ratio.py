"""Ratios beyond fp32's range: r adv is 0 where the advantage is, and the clamped term alone where that is above 0."""
import numpy as np
import pytest
import torch

import policy_loss_ref as R
import test_gpu_policy_loss as L
from policy_loss_bounds import bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("ref", ["logits", "logp", "none"])
@pytest.mark.parametrize("A", [6, 48, 100, 1500, 9001])
def test_actions_that_the_collecting_policy_hardly_took(A, ref, dtype):
    d = L.make(8, A, dtype, ref, seed=A, actions=torch.int64)
    torch.manual_seed(0)
    d["actions"] = torch.randint(0, A, (8,), device="cuda")
    lp = torch.log_softmax(d["logits"].double(), 1).gather(1, d["actions"][:, None])[:, 0]
    d["old_logp"] = (lp + 0.1).float()
    if ref == "logp":
        d["ref_logp"] = (lp + 0.2).float()
    d["old_logp"][1], d["advantages"][1] = -200.0, 0.0
    d["old_logp"][2], d["advantages"][2] = -3e38, 0.0
    d["old_logp"][3], d["advantages"][3] = -200.0, 1.5      # (clipped: the gradient of the action's term is 0)
    a = {k: L.to64(v) for k, v in dict(x=d["logits"], actions=d["actions"], old_logp=d["old_logp"], adv=d["advantages"],
                                       ref_logits=d["ref_logits"], ref_logp=d["ref_logp"]).items()}
    a["old_logp"] = np.maximum(a["old_logp"], -300.0)       # (e^300 is beyond fp32 and within fp64)
    want = R.loss(**a, **L.COEF)
    # For the bounds a clipped row's ratio is one within fp32: nothing of its loss or gradient depends on it.
    near = dict(a, old_logp=np.where(a["old_logp"] <= -200, L.to64(lp) - 1, a["old_logp"]))
    tol = bounds(**near, **L.COEF, want=want, half_step=2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24)
    got = L.run(d)
    for n, ref_n, t in zip(("stats", "logp", "dlogits"), want, tol):
        assert (np.abs(L.to64(got[n]) - ref_n) <= t).all(), n
    d["old_logp"][1] = -float("inf")                        # not a ratio at all
    got = L.run(d)
    assert torch.isnan(got["stats"][0]) and torch.isnan(got["dlogits"][1].float()).any()
    d["old_logp"][1], d["old_logp"][2] = 0.0, float("nan")
    got = L.run(d)
    assert torch.isnan(got["stats"][0]) and torch.isnan(got["dlogits"][2].float()).any()
