"""A small spiking network learns from a larger one and answers by drawing.

    python examples/distill.py [--steps 200] [--teacher-steps 200] [--batch 64] [--hidden 64]

The teacher (two LIF layers) trains on class-conditional latency codes with labels. Then, batch by batch, its readout's
K largest logits at every step are recorded (snn_readout_top) and a student with one small hidden layer trains on the
labels and on the record (snn_readout_distill beside snn_readout_ce, the sparse backward from both). At the end both
answer a fresh batch from one step's membrane, by the largest logit and by a draw with temperature, top-k, top-p and min-p
(snn_readout_sample). Prints the losses and how often the answers are the label.
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2105_08810_amd import pipeline  # noqa: E402
from synth import CONFIGS, make_inputs  # noqa: E402
from synth.inputs import make_labels, make_spikes  # noqa: E402


def student_of(teacher: pipeline.Network, hidden: int, seed: int) -> pipeline.Network:
    """A network with one hidden LIF layer on the teacher's inputs and labels."""
    g = np.random.default_rng(seed)
    n_in, C = teacher.X.shape[2], teacher.W_out.shape[1]
    dev = teacher.X.device
    first = teacher.Ws[0]  # weights as large as the teacher's
    W = (g.standard_normal((n_in, hidden)) * float(first.std())).astype(np.float32)
    W_out = (g.standard_normal((hidden, C)) / math.sqrt(hidden)).astype(np.float32)
    return pipeline.Network(X=teacher.X, Ws=[torch.from_numpy(W).to(dev)], W_out=torch.from_numpy(W_out).to(dev),
                            alphas=teacher.alphas[:1], alpha_out=teacher.alpha_out, labels=teacher.labels,
                            loss_mode=teacher.loss_mode, theta=teacher.theta, beta=teacher.beta)


def set_batch(net: pipeline.Network, X: torch.Tensor, labels: torch.Tensor):
    net.X, net.labels = X, labels


def run(steps=200, teacher_steps=200, batch=64, hidden=64, K=4, tau=2.0, b_th=0.5, lr=1e-3, seed=0, say=print):
    cfg = CONFIGS["latency_train"]

    def data(k):
        of = list(range(k * batch, (k + 1) * batch))
        return (torch.from_numpy(make_spikes(cfg, of)).cuda(), torch.from_numpy(make_labels(cfg, of).astype("int32")).cuda())

    batches = [data(k) for k in range(4)]
    teacher = pipeline.from_inputs(make_inputs(cfg, list(range(batch))))
    opt = pipeline.Adam(teacher.params(), lr=lr)
    for k in range(teacher_steps):
        set_batch(teacher, *batches[k % 3])
        out = teacher.train_step(opt, b_th)
    say(f"teacher: cross-entropy {float(out['ce']):.4f}")
    records = []
    for X, labels in batches[:3]:
        set_batch(teacher, X, labels)
        records.append(teacher.forward().record(K, tau))
    student = student_of(teacher, hidden, seed)
    opt = pipeline.Adam(student.params(), lr=lr)
    # the membrane says little in the first steps: the first fifth of the rows has no weight
    T = student.T
    live = torch.zeros((T, batch), device="cuda")
    live[T // 5:] = tau * tau / ((T - T // 5) * batch)
    first = last = None
    for k in range(steps):
        set_batch(student, *batches[k % 3])
        out = student.train_step(opt, b_th, distill=pipeline.Distill(records[k % 3], live))
        if k < 3:
            first = float(out["kd"]) if first is None else max(first, float(out["kd"]))
    last = float(out["kd"])
    say(f"student: cross-entropy {float(out['ce']):.4f}, distillation {first:.4f} -> {last:.4f}")
    # answers on the batch that neither has seen
    X, labels = batches[3]
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(batch, generator=g, device="cuda")
    f = lambda v, d=torch.float32: torch.full((batch,), v, dtype=d, device="cuda")  # noqa: E731
    right = {}
    for name, net in (("teacher", teacher), ("student", student)):
        set_batch(net, X, labels)
        net.forward()
        step = T // 2  # the inputs fire early and the membrane leaks: its scale there sets the temperature
        best, _, _ = net.draw(u, temperature=f(0.0), step=step)
        drawn, logp, kept = net.draw(u, 0.3 * net.V_out[step].std().expand(batch).contiguous(), f(5, torch.int32),
                                     f(0.9), f(0.02), step=step)
        right[name] = (float((best == labels).float().mean()), float((drawn == labels).float().mean()))
        say(f"{name}: right by the largest logit {right[name][0]:.2f}, by a draw {right[name][1]:.2f} "
            f"(mean log-probability {float(logp.mean()):.3f}, classes kept {float(kept.float().mean()):.1f})")
    return first, last, right


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--teacher-steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=64)
    a = ap.parse_args()
    run(a.steps, a.teacher_steps, a.batch, a.hidden)
