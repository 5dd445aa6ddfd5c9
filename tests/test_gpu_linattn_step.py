"""One step of linear attention (T = 1), the serving form: lengths, resets and states in place, against the formula."""
import pytest
import torch

import test_gpu_linattn as L
from paper_2609_13716_gb300 import aht

pytestmark = pytest.mark.gpu
NAN = float("nan")


def state_at(shift, s):
    """The same values ``shift`` elements behind a 16-byte boundary."""
    t = torch.empty(s.numel() + 4, device="cuda")[shift:shift + s.numel()].view(s.shape)
    return t.copy_(s)


def step(d, state, lengths=None, reset=None):
    o = torch.full((1, *d["v"].shape[1:]), 7.0, dtype=d["v"].dtype, device="cuda")
    aht.aht_linattn_forward(d["q"], d["k"], d["v"], d["log_decay"], o, reset=reset, lengths=lengths, s0=state, s_last=state, scale=0.25)
    return o


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("N,H,K,V", [(1, 1, 1, 1), (5, 3, 64, 64), (7, 2, 50, 33), (600, 2, 33, 12), (70, 4, 128, 128), (300, 3, 16, 128)])
def test_states_in_place_at_any_boundary(N, H, K, V, shift, dtype):
    d = L.make(1, N, H, K, V, dtype, seed=61, resets=0.3)
    apart = L.run(d, backward=False)
    state = state_at(shift, d["s0"])
    o = step(d, state, reset=d["reset"])
    L.verify(dict(o=o, s_last=state), d, backward=False)
    if shift == 0 or V % 4:
        assert torch.equal(o, apart["o"]) and torch.equal(state, apart["s_last"])


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("N,H,K,V", [(6, 3, 64, 64), (6, 2, 50, 33), (700, 2, 128, 128)])
def test_envs_that_have_ended(N, H, K, V, shift, dtype):
    """lengths of 0 and below: o is 0, the state stays bit for bit, and the inputs may hold anything; above 1 is one step."""
    d = L.make(1, N, H, K, V, dtype, seed=62, resets=0)
    lengths = torch.tensor([0, 1, 5, -3], dtype=torch.int32, device="cuda").repeat(N)[:N].contiguous()
    ended = (lengths < 1).nonzero()[:, 0]
    want_state = state_at(shift, d["s0"])
    want = step(d, want_state)
    reset = torch.zeros(1, N, dtype=torch.uint8, device="cuda")
    for n in ("q", "k", "v"):
        d[n][0, ended] = NAN
    reset[0, ended] = 1
    state = state_at(shift, d["s0"])
    o = step(d, state, lengths=lengths, reset=reset)
    live = (lengths > 0).nonzero()[:, 0]
    assert torch.equal(o[0, live], want[0, live]) and torch.equal(state[live], want_state[live])
    assert (o[0, ended] == 0).all() and torch.equal(state[ended], d["s0"][ended])


@pytest.mark.parametrize("dtype", L.DTYPES)
@pytest.mark.parametrize("bad", [NAN, float("inf")])
@pytest.mark.parametrize("K,V", [(64, 64), (50, 33), (128, 128)])
def test_a_reset_drops_what_is_not_finite(K, V, bad, dtype):
    d = L.make(1, 6, 2, K, V, dtype, seed=63, resets=0)
    d["reset"] = torch.zeros(1, 6, dtype=torch.uint8, device="cuda")
    d["reset"][0, 2] = d["reset"][0, 3] = 1
    want_state = d["s0"].clone()
    want = step(d, want_state, reset=d["reset"])
    state = d["s0"].clone()
    state[2] = bad
    state[3, 1, K // 2, V // 2] = bad
    state[4, 0, K // 2, V // 2] = bad               # (no reset there)
    o = step(d, state, reset=d["reset"])
    fine = [0, 1, 2, 3, 5]
    assert torch.equal(o[:, fine], want[:, fine]) and torch.equal(state[fine], want_state[fine])
    o4, w4 = o[0, 4].float(), want[0, 4].float()
    hit = torch.zeros(2, V, dtype=torch.bool, device="cuda")
    hit[0, V // 2] = True
    assert not torch.isfinite(o4[hit]).any() and torch.equal(o4[~hit], w4[~hit])
    assert not torch.isfinite(state[4, 0, K // 2, V // 2]) and int((~torch.isfinite(state)).sum()) == 1
