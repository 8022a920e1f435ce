"""The agent's loop on a small job: a training iteration made of the library's operators, against the same iteration by torch's autograd
in fp32, and the loop through theta_sys and the goodput model."""
import numpy as np
import pytest

import oracle as O

pytestmark = pytest.mark.gpu


def test_a_micro_batch_has_the_gradient_autograd_gives():
    """bfloat16 operands and intermediate rows against fp32: each of a handful of roundings is 2^-8 of its value, of independent signs in
    sums of many; in the 2-norm a gradient stays within 2^-5."""
    import torch
    from paper_2008_12260_amd.agent import Job
    job = Job(V=500, D=64, length=16, seed=1)
    tokens = job.examples(9)
    rounded = job.parameters.bfloat16()
    got = torch.empty(rounded.shape, dtype=torch.bfloat16, device="cuda")
    loss = job.micro_batch(tokens, job.parts(rounded), got)
    leaves = [p.float().clone().requires_grad_() for p in job.parts(rounded)]
    rows = leaves[0][tokens[:, :-1].reshape(-1)] * job.scale
    logits = (rows + rows @ leaves[1].t()) @ leaves[2].t()
    want = torch.nn.functional.cross_entropy(logits, tokens[:, 1:].reshape(-1))
    want.backward()
    assert abs(float(loss) - float(want)) < 2.0 ** -6 * float(want)
    for g, leaf in zip(job.parts(got), leaves):
        assert float((g.float() - leaf.grad).norm()) <= 2.0 ** -5 * float(leaf.grad.norm())


def test_the_loop_trains_the_job_and_takes_the_goodput_models_choice():
    from paper_2008_12260_amd.agent import Job, run
    rounds = []
    state = run(Job(V=1000, D=64, length=32, rate=0.05), m0=4, m_max=32, rounds=3, iterations=10, on_round=lambda s, more: rounds.append((s.m, s.s, more)))
    assert len(rounds) == 3 and len(state.records) == 3 * 13
    assert np.mean(state.losses[-5:]) < 0.8 * np.mean(state.losses[:5])
    assert all(np.isfinite(phi) and phi > 0 for _, _, phi, _ in state.choices)
    for m, s, more in rounds:
        one = np.ones((1, 1), np.int32)
        want = O.fitness(np.ones((1, 1, 1), np.int32), more["params"], more["m_grid"], np.ones((1, 2), np.int32), one, np.ones(1, np.int32), -1.0, 30.0, 4)
        assert (m, s) == (int(want["best_m"][0, 0]), int(want["best_s"][0, 0]))
        assert more["result"]["status"] == 0


def test_the_noise_scale_of_a_job_is_that_of_its_gradients():
    import torch
    from paper_2008_12260_amd.agent import Job
    job = Job(V=300, D=32, length=8, seed=2)
    for s in (3, 0, 0):
        loss, noise, seconds = job.iteration(5, s)
        assert np.isfinite(loss) and seconds > 0
        if s == 3:
            g = job.gradients.double()
            trace = 5.0 * g.var(0).sum()
            norm = g.mean(0).square().sum() - trace / 20.0
            assert abs(noise[0] / float(trace) - 1) < 1e-9 and abs(noise[1] - float(norm)) < 1e-9 * float(trace)
    assert noise is not None and np.isfinite(noise[0]) and noise[0] > 0
