"""One round of population-based training on one GPU, learner included.

A team game's population fills its payoff table and the meta-solver mixes its
policies.  A learner then trains a best response to the mixture from
trajectory records (linear layers, clipped policy loss with a divergence from
the policy it started as) and distils the mixture's own policies into one
student from their top logits, with dropout if asked for, and from teachers held
in 4 bits if asked for.  Both join the population, and the new cells of
the table are simulated.

    python examples/learner.py [--envs N] [--steps K] [--policies P] [--dropout p] [--teacher-bits 4]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2106_07551_amd as M  # noqa: E402
import workloads as W  # noqa: E402
from paper_2106_07551_amd import workload_io as IO  # noqa: E402


class Net:
    """An MLP policy of the population's shape: fp32 weights that the optimizer
    changes, bf16 copies that the layers use.  The hidden layers run in bf16,
    the output layer in fp32 (bf16 operands, fp32 logits), as the
    population's kernels do."""

    def __init__(self, weights, biases):
        self.w = [w.clone() for w in weights]          # [out][in] fp32
        self.b = [b.clone() for b in biases]
        self.refresh()

    def refresh(self):
        self.half = [w.bfloat16() for w in self.w]

    def forward(self, obs, drop=None):
        """The logits; drop: (p, seed, step) of dropout behind the hidden layers."""
        self.x = [obs]
        self.pre = []
        self.drop = drop
        for l in range(2):
            pre = torch.empty((obs.shape[0], self.w[l].shape[0]), dtype=torch.bfloat16,
                              device="cuda")
            y = M.linear(self.x[l], self.half[l], self.b[l], act=M.ACT_RELU, pre=pre)
            if drop:
                M.dropout(y, *drop, layer=l, out=y)
            self.x.append(y)
            self.pre.append(pre)
        self.x[2] = self.x[2].float()
        return M.linear(self.x[2], self.half[2].float(), self.b[2])

    def backward(self, dlogits, rate):
        """Gradients of all layers, then one descent step of size `rate`."""
        dy, dw, db = M.linear_backward(dlogits, self.x[2], self.half[2].float())
        grads = [(dw, db)]
        dy = dy.bfloat16()
        for l in (1, 0):
            if self.drop:
                M.dropout_backward(dy, *self.drop, layer=l, dx=dy)
            dy, dw, db = M.linear_backward(dy, self.x[l], self.half[l], act=M.ACT_RELU,
                                           pre=self.pre[l], want=(l > 0, True, True))
            grads.append((dw.float(), db))
        for l, (dw, db) in zip((2, 1, 0), grads):
            self.w[l] -= rate * dw
            self.b[l] -= rate * db
        self.refresh()


class Teachers:
    """The mixture's policies, frozen: weights [policy][out][in] in bf16 or in 4 bits, all
    policies' logits in one grouped call per layer."""

    # Rows of all policies that the layers in 4 bits take as they are (us, and with the weights in
    # full width first: one policy's 512 -> 512 bf16, 2048 rows 7.7 and 11.0, 16384 38 and 22, four
    # policies' 512 rows 7.6 and 11.4, 2048 22.4 and 17.4; of 256 -> 512 the limit lies at 3000)
    FEW = 4096

    def __init__(self, weights, biases, bits=16):
        self.b = biases
        self.shapes = [w.shape[1:] for w in weights]
        self.w = [M.quantize_fp4(w) if bits == 4 else w.bfloat16() for w in weights]
        self.bits = bits

    def layer(self, l, x, act):
        if self.bits == 16:
            return M.linear(x, self.w[l].to(x.dtype), self.b[l], act=act)
        if len(self.b[l]) * x.shape[-2] <= self.FEW:
            return M.linear_fp4(x, *self.w[l], self.shapes[l][0], self.b[l], act=act)
        return M.linear(x, M.dequantize_fp4(*self.w[l], *self.shapes[l], dtype=x.dtype),
                        self.b[l], act=act)

    def logits(self, obs):
        h = obs
        for l in range(2):
            h = self.layer(l, h, M.ACT_RELU)
        return self.layer(2, h.float(), M.ACT_NONE)


def mixture_lists(teachers, obs, policy_of_row, top):
    """The top entries of each row's policy: every policy's logits on all rows, then
    each row's own (log probabilities are logits less a number of the row's, which
    distillation does not see)."""
    own = teachers.logits(obs)[policy_of_row, torch.arange(obs.shape[0], device="cuda")]
    _, idx, val = M.log_probs(own, top=top)
    return idx, val


def run(n_envs=512, horizon=8, policies=6, steps=20, top=6, rate=3.0, dropout=0.0, teacher_bits=16,
        say=print):
    wl = W.team_variant(4, d=256, P=policies, n_envs=n_envs, horizon=horizon)
    env = IO.make_env(wl)
    ws = [torch.from_numpy(w).cuda() for w in wl.weights]
    bs = [torch.from_numpy(b).cuda() for b in wl.biases]
    pop = M.Population(M.POLICY_MLP_BF16, policies, wl.n_actions, dims=list(wl.dims), weights=ws,
                       biases=bs)
    pairs = M.meta_sample(wl.sigma, policies, n_envs, wl.n_agents, wl.seed)
    pop.rollout(env, n_envs, pairs, wl.seed, horizon)
    game = pop.payoff_matrix()
    sigma, gap = M.solve_fp(game, 500)
    say(f"population of {policies}: exploitability {float(gap):.4f}")

    # --- a best response for the row side, against the column side's mixture
    row_seats = [k for k in range(wl.n_agents) if wl.team[k] > 0]
    start = Net([w[0] for w in ws], [b[0] for b in bs])
    net = Net(start.w, start.b)
    returns = []
    for step in range(steps):
        trial = M.Population(M.POLICY_MLP_BF16, policies + 1, wl.n_actions, dims=list(wl.dims),
                             weights=[torch.cat([w, v[None]]) for w, v in zip(ws, net.w)],
                             biases=[torch.cat([b, v[None]]) for b, v in zip(bs, net.b)])
        pairs = M.meta_sample_device(sigma, policies, n_envs, wl.n_agents, wl.seed + 1,
                                     seat_row=[1] * wl.n_agents)
        pairs[:, row_seats] = policies
        traj = M.Traj(n_envs * horizon, wl.n_agents, obs_shape=(wl.d,), obs_dtype=torch.bfloat16)
        trial.rollout_traj(env, n_envs, pairs, wl.seed + 2 + step, horizon, traj)
        trial.close()
        # reward to go of the row side, centred per step, one row per (step, env, seat)
        rew = traj.rewards.view(horizon, n_envs)
        returns.append(float(rew.sum(0).mean()))
        togo = rew.flip(0).cumsum(0).flip(0)
        adv = (togo - togo.mean(1, keepdim=True)) / (togo.std(1, keepdim=True) + 1e-6)
        seat = row_seats[step % len(row_seats)]
        actions = traj.actions[:, seat].contiguous()
        adv = adv.reshape(-1).contiguous()
        ref_logits = start.forward(traj.obs)
        old = None
        for _ in range(2):
            logits = net.forward(traj.obs)
            if old is None:   # log probabilities under the policy that acted
                old = M.log_probs(logits, actions)[0][0]
            total, stats, dlogits = M.policy_loss(logits, actions, old, adv, kl_coef=0.02,
                                                  entropy_coef=0.002, ref_logits=ref_logits)
            net.backward(dlogits, rate)
    say(f"best response: mean return {returns[0]:.4f} -> {returns[-1]:.4f}, "
        f"divergence from its start {float(stats[2].mean()):.4f}, "
        f"entropy {float(stats[3].mean()):.4f}")

    # --- the mixture distilled into one policy, on the last records
    obs = traj.obs
    teacher = M.meta_sample_device(sigma, policies, obs.shape[0], 2, wl.seed + 99,
                                   seat_row=[0, 0])[:, 0].long()
    idx, val = mixture_lists(Teachers(ws, bs, teacher_bits), obs, teacher, top)
    student = Net([w.mean(0) for w in ws], [b.mean(0) for b in bs])
    losses = []
    for step in range(steps):
        drop = (dropout, wl.seed, step) if dropout else None
        total, _, dlogits = M.distill_loss(student.forward(obs, drop), idx, val, temperature=2.0)
        student.backward(dlogits, rate)
        losses.append(float(total))
    say(f"student: distillation loss {losses[0]:.4f} -> {losses[-1]:.4f}")

    # --- both join the population; only the new cells are simulated
    pop.extend(2, weights=[torch.stack([a, b]) for a, b in zip(net.w, student.w)],
               biases=[torch.stack([a, b]) for a, b in zip(net.b, student.b)])
    new = M.expansion_pairs(policies + 2, policies, 4, wl.n_agents, team=list(wl.team))
    pop.rollout(env, new.shape[0], new, wl.seed, horizon, env_offset=n_envs)
    game = pop.payoff_matrix()
    sigma, gap = M.solve_fp(game, 500)
    say(f"population of {policies + 2}: exploitability {float(gap):.4f}, "
        f"weight of the best response {float(sigma[0, policies] / sigma[0].sum()):.3f}, "
        f"of the student {float(sigma[0, policies + 1] / sigma[0].sum()):.3f}")
    table = pop.payoff()
    pop.close()
    return {"returns": returns, "losses": losses, "stats": stats, "table": table,
            "sigma": sigma}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--envs", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--policies", type=int, default=6)
    ap.add_argument("--dropout", type=float, default=0.0)
    ap.add_argument("--teacher-bits", type=int, choices=(4, 16), default=16)
    a = ap.parse_args()
    run(n_envs=a.envs, steps=a.steps, policies=a.policies, dropout=a.dropout,
        teacher_bits=a.teacher_bits)
