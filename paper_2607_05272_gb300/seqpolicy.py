"""A policy with memory on the simulator, made of the library's sequence operators.

The paper's agents see one observation at a time (Sec. 4.2).  This one carries a state through an
episode: per decision

    z1, y1 = dropout_add_norm(W_in obs)                       (no residual)
    x, gate = halves of W_p y1
    h = gated_scan(x, gate), dropped where an episode ends
    z2, y2 = dropout_add_norm(W_o h, residual z1)
    logits = W_h y2

Rollouts take the single-token forms, the state updated in place; updates take whole time-major
buffers [H][E], as ``rollout_collect`` lays them out.  ``update`` is one step of the clipped policy
loss with a KL term to the policy that collected the rollout; ``preference_update`` is one step of the
preference loss on pairs of envs, the one with the larger return preferred.  Actions are sampled without
dropout and every update draws a mask of its own, so it evaluates the parameters that collected the
rollout under that mask too: ratios, KL terms and margins compare parameters, not masks.  Every nonlinear
step, both losses, all their gradients and Adam run in the library's kernels; the matrix products between
them are ``torch.matmul``.

Command line: ``python -m paper_2607_05272_gb300.seqpolicy --workload c3s --iters 80``.
"""
from __future__ import annotations

import argparse
import json

import torch

from . import simx
from . import workloads as W


class SeqPolicy:
    """Parameters in one flat fp32 vector with views; buffers for E envs and H decisions."""

    def __init__(self, obs_dim: int, n_actions: int, envs: int, horizon: int, width: int = 64,
                 p: float = 0.05, seed: int = 1):
        self.D, self.A, self.E, self.H, self.C = obs_dim, n_actions, envs, horizon, width
        self.p, self.seed = p, seed
        c = width
        shapes = dict(w_in=(c, obs_dim), gain1=(c,), w_p=(2 * c, c), bias=(c,), w_o=(c, c),
                      gain2=(c,), w_h=(n_actions, c))
        # every parameter starts on a 16-byte boundary
        sizes = {k: (torch.Size(s).numel() + 3) // 4 * 4 for k, s in shapes.items()}
        n = sum(sizes.values())
        self.flat = torch.zeros(n, device="cuda")
        self.grad_flat = torch.zeros(n, device="cuda")
        self.w, self.g, off = {}, {}, 0
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for k, s in shapes.items():
            m = torch.Size(s).numel()
            self.w[k] = self.flat[off:off + m].view(s)
            self.g[k] = self.grad_flat[off:off + m].view(s)
            off += sizes[k]
            if k.startswith("w_"):
                scale = (0.1 if k == "w_h" else 1.0) * s[1] ** -0.5
                self.w[k].copy_(torch.randn(s, generator=gen, device="cuda") * scale)
            elif k.startswith("gain"):
                self.w[k].fill_(1.0)
            else:
                self.w[k].fill_(2.0)  # gates that remember about eight decisions
        self.m, self.v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        self.t = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.gen = gen
        self.calls = 0  # updates so far: the dropout's step

        def ws(size):
            return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        rows = horizon * envs
        self.scan_ws = ws(simx.gated_scan_workspace_size(envs, horizon, c))
        self.norm_ws = ws(simx.dropout_add_norm_grad_workspace_size(rows, c))
        self.loss_ws = ws(simx.token_loss_grad_workspace_size(rows))
        self.pref_ws = ws(simx.preference_loss_grad_workspace_size(rows, envs // 2))
        self.adam_ws = ws(simx.adam_workspace_size(n))
        self.stats = torch.empty(5, device="cuda")
        self.pref_stats = torch.empty(3, device="cuda")

    # ------------------------------------------------------------------ forward

    def step(self, obs, state):
        """Logits [E, A] of one decision from obs [E, D]; the state [E, C] is updated in place."""
        w, e, c = self.w, obs.shape[0], self.C
        z1 = obs @ w["w_in"].t()
        y1 = torch.empty_like(z1)
        simx.dropout_add_norm(z1, w["gain1"], y1)
        pr = (y1 @ w["w_p"].t()).view(e, 1, 2 * c)
        h = torch.empty((e, 1, c), device="cuda")
        simx.gated_scan(pr[:, :, :c], pr[:, :, c:], h, bias=w["bias"], h0=state, h_last=state)
        o, y2 = h.view(e, c) @ w["w_o"].t(), y1
        simx.dropout_add_norm(o, w["gain2"], y2, residual=z1)
        return y2 @ w["w_h"].t()

    def views(self, flat) -> dict:
        """The parameters by name in a vector laid out as `flat`."""
        return {k: flat[v.storage_offset():v.storage_offset() + v.numel()].view(v.shape) for k, v in self.w.items()}

    def forward(self, obs, done, state, p: float, step: int, w=None) -> dict:
        """The pass over a rollout: obs [H, E, D], done [H, E], state [E, C] before its first
        decision; w: other parameters than the policy's own.  Returns what the backward pass takes,
        logits [H * E, A] among it."""
        w, c, (hh, e, d) = w or self.w, self.C, obs.shape
        n = hh * e
        f = dict(obs=obs.reshape(n, d), done=done.t(), state=state, p=p, step=step, shape=(hh, e))

        def empty(*shape):
            return torch.empty(shape, device="cuda")
        u = f["obs"] @ w["w_in"].t()
        f["z1"], f["y1"], f["r1"] = empty(n, c), empty(n, c), empty(n)
        simx.dropout_add_norm(u, w["gain1"], f["y1"], z=f["z1"], rstd=f["r1"], p=p, seed=self.seed,
                              step=2 * step)
        pr = (f["y1"] @ w["w_p"].t()).view(hh, e, 2 * c).transpose(0, 1)
        f["x"], f["gate"] = pr[:, :, :c], pr[:, :, c:]
        f["h"] = empty(hh, e, c).transpose(0, 1)
        simx.gated_scan(f["x"], f["gate"], f["h"], self.scan_ws, bias=w["bias"], h0=state,
                        done=f["done"])
        o = f["h"].transpose(0, 1).reshape(n, c) @ w["w_o"].t()
        f["z2"], f["y2"], f["r2"] = empty(n, c), empty(n, c), empty(n)
        simx.dropout_add_norm(o, w["gain2"], f["y2"], residual=f["z1"], z=f["z2"], rstd=f["r2"],
                              p=p, seed=self.seed, step=2 * step + 1)
        f["logits"] = f["y2"] @ w["w_h"].t()
        return f

    def backward(self, f: dict, dlogits):
        """Fills the gradient vector from the logits' gradient."""
        w, g, c, (hh, e) = self.w, self.g, self.C, f["shape"]
        n = hh * e

        def empty():
            return torch.empty((n, c), device="cuda")
        torch.matmul(dlogits.t(), f["y2"], out=g["w_h"])
        dy2 = dlogits @ w["w_h"]
        do, dz1 = empty(), empty()
        simx.dropout_add_norm_grad(f["z2"], w["gain2"], f["r2"], dy2, do, self.norm_ws, dresidual=dz1,
                                   dgain=g["gain2"], p=f["p"], seed=self.seed, step=2 * f["step"] + 1)
        h_rows = f["h"].transpose(0, 1).reshape(n, c)
        torch.matmul(do.t(), h_rows, out=g["w_o"])
        dh = (do @ w["w_o"]).view(hh, e, c).transpose(0, 1)
        dpr = torch.empty((hh, e, 2 * c), device="cuda")
        dv = dpr.transpose(0, 1)
        simx.gated_scan_grad(f["x"], f["gate"], f["h"], dh, dv[:, :, :c], dv[:, :, c:], self.scan_ws,
                             bias=w["bias"], h0=f["state"], done=f["done"], dbias=g["bias"])
        dpr = dpr.view(n, 2 * c)
        torch.matmul(dpr.t(), f["y1"], out=g["w_p"])
        dy1 = dpr @ w["w_p"]
        du = empty()
        simx.dropout_add_norm_grad(f["z1"], w["gain1"], f["r1"], dy1, du, self.norm_ws, dz=dz1,
                                   dgain=g["gain1"], p=f["p"], seed=self.seed, step=2 * f["step"])
        torch.matmul(du.t(), f["obs"], out=g["w_in"])

    # ------------------------------------------------------------------ rollouts and updates

    def rollout(self, sim, state) -> dict:
        """H decisions of every env, sampled; the state goes on in place.  b["params"]: the parameters that
        sampled them."""
        hh, e = self.H, self.E
        b = dict(obs=torch.empty((hh, e, self.D), device="cuda"),
                 action=torch.empty((hh, e), dtype=torch.int64, device="cuda"),
                 logp=torch.empty((hh, e), device="cuda"), reward=torch.empty((hh, e), device="cuda"),
                 done=torch.empty((hh, e), dtype=torch.uint8, device="cuda"), state=state.clone(),
                 params=self.flat.clone())
        cols = torch.empty((self.D, e), device="cuda")
        sim.observe(cols)
        for t in range(hh):
            b["obs"][t] = cols.t()
            logits = self.step(b["obs"][t], state)
            noise = torch.empty_like(logits).exponential_(generator=self.gen)
            b["action"][t] = (logits - noise.log()).argmax(1)
            simx.token_loss_grad(logits, b["action"][t], None, self.stats, self.loss_ws,
                                 logp=b["logp"][t])
            sim.step("external", actions=b["action"][t].int(), obs=cols, reward=b["reward"][t],
                     done=b["done"][t])
            state.masked_fill_(b["done"][t, :, None] != 0, 0.0)
        return b

    def reference(self, b: dict, step: int):
        """Log probabilities [H, E] of a rollout's actions by the parameters that collected it, under the
        dropout mask of `step`; b["logp"] as it is where no dropout or no parameters are there."""
        if "params" not in b or self.p == 0.0:
            return b["logp"]
        f = self.forward(b["obs"], b["done"], b["state"], self.p, step, self.views(b["params"]))
        logp = torch.empty_like(b["logp"])
        simx.token_loss_grad(f["logits"], b["action"].view(-1), None, self.stats, self.loss_ws,
                             logp=logp.view(-1))
        return logp

    def _adam(self, lr):
        simx.adam_step(self.flat, self.grad_flat, self.m, self.v, self.t, lr, max_grad_norm=0.5,
                       workspace=self.adam_ws)

    def update(self, b: dict, adv, lr: float = 1e-3, clip: float = 0.2, c_kl: float = 0.02,
               c_entropy: float = 0.01):
        """One step of the clipped policy loss on a rollout with advantages [H, E]; the KL term is to
        the policy that collected it.  Returns the loss's statistics (device)."""
        logp = self.reference(b, self.calls).view(-1)
        f = self.forward(b["obs"], b["done"], b["state"], self.p, self.calls)
        self.calls += 1
        simx.token_loss_grad(f["logits"], b["action"].view(-1), adv.reshape(-1), self.stats,
                             self.loss_ws, logp_old=logp, logp_ref=logp, clip_low=clip,
                             clip_high=clip, c_kl=c_kl, c_entropy=c_entropy, grad=f["logits"])
        self.backward(f, f["logits"])
        self._adam(lr)
        return self.stats

    def preference_update(self, b: dict, lr: float = 1e-4, beta: float = 0.1):
        """One step of the preference loss on pairs of envs (2p, 2p + 1): the sequence of the larger
        return is preferred (equal returns: neither, the pair counts for nothing), the rollout's log
        probabilities are the reference.  Returns the loss's statistics (device)."""
        hh, e = self.H, self.E // 2 * 2
        ret = b["reward"].sum(0)[:e].view(-1, 2)
        swap = (ret[:, 1] > ret[:, 0]).long()[:, None]
        weight = (ret[:, 1] != ret[:, 0]).float() / max(len(ret), 1)
        pair = torch.arange(e, device="cuda").view(-1, 2)
        order = torch.cat([pair.gather(1, swap), pair.gather(1, 1 - swap)], 1).view(-1)
        logp = self.reference(b, self.calls)
        f = self.forward(b["obs"], b["done"], b["state"], self.p, self.calls)
        self.calls += 1

        def rows(x):  # [H, E, ...] time-major rows as whole sequences, the preferred one first
            return x.transpose(0, 1)[order].reshape((e * hh,) + x.shape[2:])
        logits = rows(f["logits"].view(hh, self.E, self.A))
        start = torch.arange(e + 1, device="cuda") * hh
        simx.preference_loss_grad(logits, rows(b["action"]), start, self.pref_stats, self.pref_ws,
                                  logp_ref=rows(logp), weight=weight, beta=beta, grad=logits)
        dlogits = torch.zeros((self.E, hh, self.A), device="cuda")
        dlogits[order] = logits.view(e, hh, self.A)
        self.backward(f, dlogits.transpose(0, 1).reshape(hh * self.E, self.A))
        self._adam(lr)
        return self.pref_stats


def train(workload: str = "c3s", envs: int = 1024, horizon: int = 128, iters: int = 80,
          epochs: int = 4, width: int = 64, lr: float = 3e-3, gamma: float = 0.99, seed: int = 1,
          every: int = 10, preferences: int = 10) -> list:
    """Trains on a workload; every `preferences` iterations (0: never) one preference step on top.
    Returns one dict per iteration."""
    cfg = W.CONFIGS[workload](envs)
    dims, has_value = W.mlp_dims(workload)
    sim = simx.Sim(cfg)
    sim.reset(seed)
    pol = SeqPolicy(sim.D, dims[-1] - int(has_value), envs, horizon, width, seed=seed)
    state = torch.zeros((envs, width), device="cuda")
    n = envs * horizon
    ret, adv = torch.empty((horizon, envs), device="cuda"), torch.empty((horizon, envs), device="cuda")
    mean = torch.empty(1, device="cuda")
    base_ws = torch.empty(simx.returns_baseline_workspace_size(n), dtype=torch.uint8, device="cuda")
    hist, ps = [], torch.zeros(3, device="cuda")
    for i in range(iters):
        b = pol.rollout(sim, state)
        simx.compute_returns_gae(b["reward"], b["done"], gamma, -1.0, ret)
        simx.returns_baseline(ret, adv, mean, base_ws)
        adv /= adv.std() + 1e-6
        for _ in range(epochs):
            st = pol.update(b, adv, lr)
        if preferences and (i + 1) % preferences == 0:
            ps = pol.preference_update(b)
        s, q = st.tolist(), ps.tolist()
        hist.append({"iter": i + 1, "mean_reward": b["reward"].mean().item(), "loss": s[0],
                     "kl": s[2], "entropy": s[3], "clipped": s[4], "preference_loss": q[0],
                     "preferred": q[1]})
        if every and ((i + 1) % every == 0 or i == 0):
            print(json.dumps(hist[-1]), flush=True)
    sim.close()
    return hist


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="c3s")
    ap.add_argument("--envs", type=int, default=1024)
    ap.add_argument("--horizon", type=int, default=128)
    ap.add_argument("--iters", type=int, default=80)
    ap.add_argument("--epochs", type=int, default=4)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--lr", type=float, default=3e-3)
    ap.add_argument("--seed", type=int, default=1)
    ap.add_argument("--preferences", type=int, default=10, help="iterations per preference step")
    a = ap.parse_args(argv)
    train(a.workload, a.envs, a.horizon, a.iters, a.epochs, a.width, a.lr, seed=a.seed,
          preferences=a.preferences)


if __name__ == "__main__":
    main()
