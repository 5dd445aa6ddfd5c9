"""What is not finite in a row of the policy loss shows in that row and in the sums, wherever it stands, and
nowhere else."""
import pytest
import torch

import test_gpu_policy_loss as L

pytestmark = pytest.mark.gpu
NAN = float("nan")


def copy(t):
    """With the same strides: rows aligned as before are summed in the same order."""
    return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device).copy_(t)


def shows(d, clean, row, where):
    got = L.run(d)
    others = torch.arange(len(d["actions"]), device="cuda") != row
    for n in ("logp", "dlogits"):
        assert torch.equal(got[n][others], clean[n][others]), (where, n)
    assert torch.isnan(got["dlogits"][row].float()).any(), where
    assert torch.isnan(got["stats"][0]), where
    return got


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("ref", ["logits", "logp", "none"])
@pytest.mark.parametrize("A", [6, 48, 65, 100, 256, 1500, 9001])
@pytest.mark.parametrize("spare", [0, 1])
def test_logits_that_are_no_numbers(A, ref, dtype, spare):
    """A whole row (a diverged network's), whole vectors at its head, middle and tail, every other vector, one element."""
    d = L.make(9, A, dtype, ref, seed=A, spare=spare, actions=torch.uint8 if A < 256 else torch.int64)
    torch.manual_seed(0)
    d["actions"] = torch.randint(0, A, (9,), device="cuda")
    clean = L.run(d)
    j = torch.arange(A, device="cuda")
    for where, at in (("row", j >= 0), ("head", j < 8), ("middle", (j >= A // 2) & (j < A // 2 + 8)), ("tail", j >= A - 8),
                      ("half", j // 8 % 2 == 0), ("first", j == 0), ("last", j == A - 1), ("all but one", j != d["actions"][4])):
        x = copy(d["logits"])
        x[4, at] = NAN
        got = shows(dict(d, logits=x), clean, 4, where)
        assert torch.isnan(got["logp"][4]), where


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("A", [6, 48, 65, 100, 256, 1500, 9001])
@pytest.mark.parametrize("spare", [0, 1])
def test_a_reference_of_no_numbers(A, dtype, spare):
    """Also beside reference logits of -inf, and where the policy's own logit is -inf."""
    d = L.make(9, A, dtype, "logits", seed=A, spare=spare, actions=torch.int64)
    torch.manual_seed(0)
    d["actions"] = torch.randint(0, A, (9,), device="cuda")
    clean = L.run(d)
    j = torch.arange(A, device="cuda")
    for where, at in (("row", j >= 0), ("head", j < 8), ("middle", (j >= A // 2) & (j < A // 2 + 8)), ("tail", j >= A - 8),
                      ("half", j // 8 % 2 == 0), ("one", j == A // 2)):
        y = copy(d["ref_logits"])
        y[4, at] = NAN
        got = shows(dict(d, ref_logits=y), clean, 4, where)
        assert torch.equal(got["logp"][4], clean["logp"][4]) or A > 64, where   # (read again in another order)
        x = copy(d["logits"])
        x[4, at & (j != d["actions"][4])] = -float("inf")
        if where != "row":
            shows(dict(d, logits=x, ref_logits=y), clean, 4, where + ", masked")


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("A", [48, 100, 256, 1500, 9001])
def test_infinite_logits(A, dtype):
    d = L.make(9, A, dtype, "logits", seed=A, actions=torch.int64)
    torch.manual_seed(0)
    d["actions"] = torch.randint(0, A, (9,), device="cuda")
    clean = L.run(d)
    for name in ("logits", "ref_logits"):
        for at in (slice(0, 8), slice(A // 2, A // 2 + 1), slice(A - 8, A), slice(0, A)):
            t = copy(d[name])
            t[4, at] = float("inf")
            shows(dict(d, **{name: t}), clean, 4, (name, at))
