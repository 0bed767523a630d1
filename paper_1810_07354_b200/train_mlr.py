"""Multinomial logistic regression with a running checkpoint: the training step of the paper's first workload
(Sections 5.1, 5.3) and the checkpoint and recovery of its parameters, end to end on one GPU.

Every iteration draws a minibatch, computes loss and gradient of the softmax cross entropy
(:class:`~paper_1810_07354_b200.LinearCrossEntropy`), clips the gradient by its global norm
(:class:`~paper_1810_07354_b200.GradientNorm`) and takes a step.  Every ``r * full_period`` iterations the ``r`` most
changed blocks are saved (Section 4.2).  At ``fail_at`` some shards are lost and restored (Section 4.1).  Clipping bounds a
step by ``lr * max_norm``, so the perturbation of a recovery is at most that times the iterations since the lost blocks
were saved; both are reported.

    python -m paper_1810_07354_b200.train_mlr --classes 1000 --features 4096 --iterations 60
"""

from __future__ import annotations

import argparse
import json
from dataclasses import dataclass, field

import numpy as np

from . import api


@dataclass
class History:
    loss: list = field(default_factory=list)       # of every minibatch
    grad_norm: list = field(default_factory=list)  # before clipping
    saved_blocks: int = 0
    perturbation: float = 0.0  # ||x - x_recovered|| of the recovery
    perturbation_bound: float = 0.0
    lost_blocks: int = 0
    launches: int = 0


def make_data(samples: int, classes: int, features: int, seed: int = 0, device="cuda"):
    """Samples of a linear teacher: float32 features, the teacher's most likely class as label."""
    import torch

    g = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn(samples, features, device=device, generator=g)
    teacher = torch.randn(classes, features, device=device, generator=g)
    return x, (x @ teacher.T).argmax(dim=1)


def train(samples: int = 8192, classes: int = 1000, features: int = 4096, batch: int = 512, iterations: int = 60, lr: float = 5.0,
          max_norm: float = 0.05, r: float = 0.25, full_period: int = 8, n_shards: int = 8, lost_shards=(1, 5), fail_at: int = 40,
          block: int = 1024, seed: int = 0):
    """Runs the loop above; returns ``(weights, History)``."""
    import torch

    x, y = make_data(samples, classes, features, seed)
    w = torch.zeros(classes, features, device="cuda")
    dw, dh = torch.empty_like(w), torch.empty(batch, features, device="cuda")
    loss_op = api.LinearCrossEntropy(batch, classes, features, torch.float32)
    norm_op = api.GradientNorm([dw])  # clips in place
    ck = api.ScarCheckpoint(w.view(-1), n_shards=n_shards, row_elems=features, block_elems=min(block, features))
    period, k = max(1, round(r * full_period)), api.scar_k_from_r(r, ck.n_blocks)
    lost = np.zeros(n_shards, dtype=np.uint8)
    lost[list(lost_shards)] = 1
    h, losses, norms = History(), [], []
    order = torch.Generator(device="cuda").manual_seed(seed + 1)
    for it in range(1, iterations + 1):
        at = torch.randint(0, samples, (batch,), device="cuda", generator=order)
        loss, _, _, _ = loss_op.loss_and_grad(x[at], w, y[at], dh=dh, dw=dw)
        norms.append(norm_op.clip(max_norm))
        w.sub_(dw, alpha=lr)
        losses.append(loss)
        if it % period == 0:
            h.saved_blocks += int(ck.priority_save_k(k).k)
        if it == fail_at:
            info = ck.recover_partial(lost)
            h.perturbation, h.lost_blocks = float(info.l2), int(info.lost_blocks)
            h.perturbation_bound = lr * max_norm * it  # no step is longer than lr * max_norm
    h.loss, h.grad_norm = [float(v) for v in losses], [float(v) for v in norms]
    h.launches = api.scar_xent_launch_count(loss_op.op) + api.scar_gnorm_launch_count(norm_op.op) + api.scar_ckpt_launch_count(ck.ctx)
    for op in (loss_op, norm_op, ck):
        op.close()
    return w, h


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("samples", 8192), ("classes", 1000), ("features", 4096), ("batch", 512), ("iterations", 60), ("fail-at", 40), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=default)
    for name, default in (("lr", 5.0), ("max-norm", 0.05), ("r", 0.25)):
        ap.add_argument(f"--{name}", type=float, default=default)
    a = ap.parse_args(argv)
    _, h = train(a.samples, a.classes, a.features, a.batch, a.iterations, a.lr, a.max_norm, a.r, fail_at=a.fail_at, seed=a.seed)
    print(json.dumps({"loss_first": h.loss[0], "loss_last": h.loss[-1], "grad_norm_last": h.grad_norm[-1], "saved_blocks": h.saved_blocks,
                      "lost_blocks": h.lost_blocks, "perturbation": h.perturbation, "perturbation_bound": h.perturbation_bound,
                      "kernel_launches": h.launches}))


if __name__ == "__main__":
    main()
