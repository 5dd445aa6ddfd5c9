"""kl_coef = 0: KL is a figure of the statistics alone, and an infinite one does not reach the loss or its gradient."""
import numpy as np
import pytest
import torch

import policy_loss_ref as R
import test_gpu_policy_loss as L
from paper_2609_13716_gb300 import aht

pytestmark = pytest.mark.gpu


def run(d, ref):
    M, A = d["logits"].shape
    ws = torch.empty(aht.aht_policy_loss_workspace(M, A), dtype=torch.uint8, device="cuda")
    out = dict(stats=torch.empty(6, device="cuda"), logp=torch.empty(M, device="cuda"), dlogits=torch.empty_like(d["logits"]))
    aht.aht_policy_loss(d["logits"], d["actions"], d["old_logp"], d["advantages"], out["stats"], dlogits=out["dlogits"],
                        logp=out["logp"], workspace=ws, ent_coef=0.01, **ref)
    return out


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("M,A", [(40, 6), (200, 6), (40, 48), (40, 100), (9, 1500), (5, 9001)])
def test_the_loss_is_the_one_without_a_reference(M, A, dtype):
    d = L.make(M, A, dtype, "logits", seed=M + A, actions=torch.int64)
    torch.manual_seed(M + A)
    d["actions"] = torch.randint(0, A, (M,), device="cuda")
    want = run(d, {})
    y = d["ref_logits"].clone()
    y[1, A // 2] = y[3, :2] = -float("inf")     # the reference leaves actions out that the policy takes
    none = torch.full((M,), -1.0, device="cuda")
    none[2] = -float("inf")
    stats = R.loss(*(L.to64(d[n]) for n in ("logits", "actions", "old_logp", "advantages")), ent_coef=0.01)[0]
    for ref in (dict(ref_logits=y), dict(ref_logits=d["ref_logits"]), dict(ref_logp=none)):
        got = run(d, ref)
        assert bool(torch.isinf(got["stats"][2])) == (ref.get("ref_logits") is not d["ref_logits"])
        # (rows are summed in the same or another order: 2^-20 of sums and their logarithms, half a step more in bf16.  A ratio
        # is off, relative to itself, by what logp is off: a sum of ratios by that times its own size, above 1 where the
        # actions are not the ones that old_logp is of.)
        eps = 2.0 ** -20 * (1 + A ** 0.5 / 8)
        step = 2.0 ** -7 if dtype is torch.bfloat16 else 0
        part = [0, 1, 3, 4, 5]
        assert (np.abs(L.to64(got["stats"])[part] - stats[part]) <= 40 * eps * np.maximum(1, np.abs(stats[part]))).all()
        a, b = got["dlogits"].double(), want["dlogits"].double()
        assert bool(((a - b).abs() <= (step + 20 * eps) * b.abs() + 20 * eps / M * torch.softmax(d["logits"].double(), 1)).all())
        assert bool(((got["logp"] - want["logp"]).abs() <= 20 * eps).all())
