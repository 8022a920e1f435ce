"""The agent's half of the method on a real job (Pollux, arXiv 2008.12260, Sec. 4.1 and 4.3): a small language model trains on one
GPU with this library's operators; its gradients give the noise scale phi_t, its iterations the records that theta_sys is
fitted to, and the goodput model built from both picks the per-GPU batch size m and accumulation steps s that it trains at next.

One iteration of m examples by s + 1 micro-batches: rows looked up by token (embed), a residual layer (torch's matrix products: a job's
own layers are its own), the loss over the vocabulary and its gradients (token_loss, token_loss_grad), the table's gradient
(embed_grad); then the noise scale and the mean of the micro-batches' gradients in one pass (noise_scale; with s = 0 of this
iteration's gradient and the one before it), and the update: orthogonalised for the layer (orthogonalize), a step of fixed length for
the tables.

`Job` is what a user would have of a training program; `run` is the loop that closes with pollux_fit_theta and pollux_fitness.
"""
from __future__ import annotations

import time
from dataclasses import dataclass, field

import numpy as np

from . import NPARAM, PARAM_PHI, FitnessCall, embed, embed_grad, fit_theta, noise_scale, orthogonalize, token_loss, token_loss_grad

PARAM_M0, PARAM_M_MAX, PARAM_WEIGHT, PARAM_AGE, PARAM_M_MEM = 8, 9, 10, 11, 13      # rows of job_params (PX_M0, ...)


class Job:
    """A language model of a looked-up table [V, D], a residual layer [D, D] and a projection [V, D], in bfloat16 with fp32
    parameters, on synthetic text: each token follows from the one before it in nine of ten cases."""

    def __init__(self, V=4096, D=256, length=64, rate=0.02, seed=0):
        import torch
        if D % 8:
            raise ValueError("rows of whole 16-byte groups: D is a multiple of 8")
        self.torch, self.V, self.D, self.length, self.rate = torch, V, D, length, rate
        self.rng = torch.Generator("cuda").manual_seed(seed)
        self.after = torch.randperm(V, generator=self.rng, device="cuda")
        self.scale = float(D) ** 0.5
        sizes = (V * D, D * D, V * D)
        self.parameters = torch.randn(sum(sizes), generator=self.rng, device="cuda") * D ** -0.5
        self.parameters[:sizes[0]] *= D ** -0.5 * 4
        self.shapes, self.sizes = ((V, D), (D, D), (V, D)), sizes
        self.gradients = torch.empty((0, sum(sizes)), dtype=torch.bfloat16, device="cuda")
        self.before = None                   # the gradient of the iteration before, while m is the same
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")       # what the operators report of the tokens

    def parts(self, flat):
        """(table, layer, projection) of a flat vector, as views."""
        return [x.view(s) for x, s in zip(flat.split(self.sizes), self.shapes)]

    def examples(self, m):
        """m sequences of length + 1 tokens."""
        torch = self.torch
        tokens = torch.empty((m, self.length + 1), dtype=torch.int64, device="cuda")
        tokens[:, 0] = torch.randint(0, self.V, (m,), generator=self.rng, device="cuda")
        other = torch.randint(0, self.V, (m, self.length), generator=self.rng, device="cuda")
        strays = torch.rand((m, self.length), generator=self.rng, device="cuda") < 0.1
        for i in range(self.length):
            tokens[:, i + 1] = torch.where(strays[:, i], other[:, i], self.after[tokens[:, i]])
        return tokens

    def micro_batch(self, tokens, model, gradient):
        """Mean loss of a micro-batch; its gradient goes into `gradient`, a flat vector."""
        torch = self.torch
        table, layer, projection = model
        d_table, d_layer, d_projection = self.parts(gradient)
        x, y = tokens[:, :-1].reshape(-1), tokens[:, 1:].reshape(-1)
        rows = embed(x, table, self.scale, status=self.status)
        hidden = torch.addmm(rows, rows, layer.t())
        loss, lse = token_loss(hidden, projection, y, status=self.status)
        weight = torch.full_like(loss, 1.0 / loss.numel())
        d_hidden, _ = token_loss_grad(hidden, projection, y, lse, weight, weight_grad=d_projection)
        torch.mm(d_hidden.t(), rows, out=d_layer)
        embed_grad(x, torch.addmm(d_hidden, d_hidden, layer), self.V, self.scale, table_grad=d_table)
        return loss.mean()

    def iteration(self, m, s):
        """One iteration of s + 1 micro-batches of m examples: (mean loss, [tr(Sigma), |g|^2, phi] or None where there is a single
        gradient and none before it, seconds)."""
        torch = self.torch
        batches = [self.examples(m) for _ in range(s + 1)]
        rows = max(2, s + 1)
        if self.gradients.shape[0] != rows:
            self.gradients, self.before = torch.empty((rows, self.parameters.numel()), dtype=torch.bfloat16, device="cuda"), None
        torch.cuda.synchronize()
        began = time.perf_counter()
        model = self.parts(self.parameters.bfloat16())
        losses = [self.micro_batch(batch, model, self.gradients[i]) for i, batch in enumerate(batches)]
        if s > 0:
            mean, noise = noise_scale(self.gradients, float(m))
        else:
            noise = noise_scale(self.gradients, float(m), want_mean=False)[1] if self.before == m else None
            mean = self.gradients[0].float()
            self.gradients[1].copy_(self.gradients[0])
        self.before = m if s == 0 else None
        for k, (p, g) in enumerate(zip(self.parts(self.parameters), self.parts(mean))):
            p.sub_(orthogonalize(g) if k == 1 else g * (self.D ** -0.5 / (g.square().mean().sqrt() + 1e-20)), alpha=self.rate)
        torch.cuda.synchronize()
        seconds = time.perf_counter() - began
        if int(self.status):
            self.status.zero_()
            raise ValueError(f"a token is neither -1 nor one of the {self.V} entries of the vocabulary")
        return float(torch.stack(losses).mean()), None if noise is None else noise.cpu().numpy(), seconds


@dataclass
class AgentState:
    m: int
    s: int
    records: list = field(default_factory=list)          # (m, s, seconds)
    noise: list = field(default_factory=list)            # [tr(Sigma), |g|^2, phi] of each estimate
    losses: list = field(default_factory=list)
    choices: list = field(default_factory=list)          # (m, s, phi, theta) of every round


def choose(job_params, m_grid, Gs):
    """(m*, s*) of Eq. 13 for one job on one GPU."""
    import torch
    one = np.ones((1, 1), np.int32)
    call = FitnessCall(1, 1, 1, m_grid.shape[1], Gs, job_params, m_grid, np.ones((1, 2), np.int32), one, np.ones(1, np.int32))
    call.run(torch.ones((1, 1, 1), dtype=torch.int32, device="cuda"), outputs="all")
    got = call.results()
    return int(got["best_m"][0, 0]), int(got["best_s"][0, 0]), got


def run(job, m0=8, m_max=64, Gm=16, Gs=4, rounds=3, iterations=12, on_round=None):
    """`rounds` times: `iterations` iterations at (m, s), and one at a few others so that the throughput model sees more than one point;
    then the noise scale averaged over the round, theta_sys fitted to all records, and the next (m, s).  Returns the AgentState."""
    state = AgentState(m=m0, s=1)
    m_grid = np.unique(np.geomspace(max(1, m0 // 2), m_max, Gm).round().astype(np.int32))[None]
    job.iteration(m0, 1)                       # first use of every kernel is no record
    for _ in range(rounds):
        estimates = []
        around = [(state.m, state.s)] * iterations + [(max(1, state.m // 2), 1), (min(m_max, 2 * state.m), 0), (state.m, Gs - 1)]
        for m, s in around:
            loss, noise, seconds = job.iteration(m, s)
            state.records.append((m, s, seconds))
            state.losses.append(loss)
            if noise is not None and np.isfinite(noise).all():
                estimates.append(noise)
        state.noise += estimates
        # both parts averaged before the division: each is unbiased, their quotient is not
        trace, norm = np.mean([e[0] for e in estimates]), np.mean([e[1] for e in estimates])
        phi = float(trace / max(norm, 1e-6 * trace))
        m, s, seconds = (np.array(c)[None] for c in zip(*state.records))
        fitted = fit_theta(dict(count=np.array([m.shape[1]]), K=np.ones_like(m), nodes=np.ones_like(m), m=m, s=s, T=seconds))
        params = np.zeros((NPARAM, 1))
        params[:7] = fitted["theta"]
        params[PARAM_PHI], params[PARAM_M0], params[PARAM_M_MAX], params[PARAM_WEIGHT] = phi, m0, m_max * Gs, 1.0
        params[PARAM_AGE], params[PARAM_M_MEM] = 3600.0, m_max
        state.m, state.s, result = choose(params, m_grid, Gs)
        state.choices.append((state.m, state.s, phi, fitted["theta"][:, 0]))
        if on_round is not None:
            on_round(state, dict(params=params, m_grid=m_grid, result=result, rmsle=float(fitted["rmsle"][0])))
    return state


if __name__ == "__main__":
    def report(state, more):
        m, s, phi, theta = state.choices[-1]
        print(f"loss {np.mean(state.losses[-8:]):.3f}  phi {phi:.0f}  T_grad = {1e3 * theta[0]:.2f} ms + {1e6 * theta[1]:.1f} us m "
              f"(rmsle {more['rmsle']:.3f})  next m = {m}, s = {s}", flush=True)
    run(Job(), rounds=6, iterations=20, on_round=report)
