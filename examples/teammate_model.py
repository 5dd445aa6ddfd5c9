"""A recurrent model of the teammate, trained on collected episodes.

An LBF 7x7 ego plays the twelve rule-based teammates (aht_rollout); a gated recurrence over
the ego's observations, cleared where an episode begins, predicts the teammate's next action.
It is trained through the sequence and its gradient (aht_glr_forward, aht_glr_backward), its
matrices are updated by the orthogonalised update (aht_muon_step), its vectors and output layer
by torch's Adam, and it then serves one step at a time (aht_glr_forward with T = 1).

    python examples/teammate_model.py [--updates 40] [--envs 512] [--steps 64] [--dtype bf16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_13716_gb300 import aht, recurrent  # noqa: E402
from paper_2609_13716_gb300 import workloads as W  # noqa: E402

WIDTH = 128


class TeammateModel:
    def __init__(self, obs_dim, n_actions, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        mat = lambda r, c: (torch.randn(r, c, device="cuda", generator=g) / c ** 0.5).requires_grad_()  # noqa: E731
        vec = lambda n: torch.zeros(n, device="cuda", requires_grad=True)  # noqa: E731
        self.dtype = dtype
        self.enc, self.enc_b = mat(WIDTH, obs_dim), vec(WIDTH)
        self.proj, self.proj_b = mat(3 * WIDTH, WIDTH), vec(3 * WIDTH)
        self.out, self.out_b = mat(n_actions, WIDTH), vec(n_actions)
        decay = torch.linspace(0.9, 0.999, WIDTH, device="cuda")         # of a fully open gate
        self.lam = torch.log(torch.expm1(-torch.log(decay) / 8)).requires_grad_()
        self.matrices = [self.enc, self.proj]
        self.rest = [self.enc_b, self.proj_b, self.out, self.out_b, self.lam]

    def inputs(self, obs):
        """u8 observations [..., obs_dim] -> x, r, i [..., WIDTH]: slices of one projection."""
        u = torch.relu(obs.float() @ self.enc.t() + self.enc_b)
        return (u @ self.proj.t() + self.proj_b).to(self.dtype).split(WIDTH, dim=-1)

    def logits(self, h):
        return torch.relu(h.float()) @ self.out.t() + self.out_b

    def sequence(self, obs, reset, state):
        h, last = recurrent.gated_recurrence(*self.inputs(obs), self.lam, state, reset)
        return self.logits(h), last.detach()

    @torch.no_grad()
    def step(self, obs, reset, state):
        return self.logits(recurrent.gated_step(*self.inputs(obs), self.lam, state, reset))


def main(updates=40, envs=512, steps=64, dtype="bf16", verbose=True):
    wl = W.WORKLOADS["lbf7x7_64x50_fp32"]
    pop = [[(torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()) for w, b in p] for p in W.population(wl)]
    ctx = aht.aht_create(wl.env, pop, envs, wl.env_seed, has_value_head=list(wl.value_head), weight_dtype=aht.AHT_FP32)
    rules = [-1 - k for k in range(12)]
    model = TeammateModel(wl.env.obs_dim, wl.env.n_actions, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype])
    muon = recurrent.OrthogonalOptimizer(model.matrices, lr=0.02)
    adam = torch.optim.Adam(model.rest, lr=2e-3)
    traj = aht.traj_buffers(ctx, steps)
    # every call draws the teammates anew, so each one starts from a cleared state
    state = torch.zeros(envs, WIDTH, device="cuda")
    first = torch.ones(1, envs, dtype=torch.uint8, device="cuda")
    losses = []
    for k in range(updates):
        aht.aht_rollout(ctx, 0, rules, steps, traj)
        reset = torch.cat([first, traj["dones"][:-1]])
        logits, _ = model.sequence(traj["obs"], reset, state)
        loss = torch.nn.functional.cross_entropy(logits.flatten(0, 1), traj["tm_actions"].long().flatten())
        adam.zero_grad()
        loss.backward()
        muon.step()
        adam.step()
        losses.append(loss.detach())
        if verbose and k % 10 == 0:
            print(f"update {k}: loss {float(losses[-1]):.4f}")
    muon.sync()
    aht.aht_glr_sync()
    # the same episodes, one step at a time
    with torch.no_grad():
        whole, last = model.sequence(traj["obs"], reset, state)
    live = state.clone()
    each = torch.stack([model.step(traj["obs"][t], reset[t], live) for t in range(steps)])
    acc = float((whole.argmax(-1) == traj["tm_actions"]).float().mean())
    gap = float((whole - each).abs().max())
    aht.aht_sync(ctx)
    if verbose:
        print(f"loss {float(losses[0]):.4f} -> {float(losses[-1]):.4f}, teammate's action predicted {acc:.3f}, "
              f"sequence against single steps: largest difference of a logit {gap:.2g}")
    return [float(v) for v in losses], acc, gap


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--updates", type=int, default=40)
    ap.add_argument("--envs", type=int, default=512)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    main(**vars(ap.parse_args()))
