"""The logistic regression example: loss and gradient, clipping, saves and a recovery together."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_1810_07354_b200 import train_mlr  # noqa: E402


def test_training_with_saves_and_a_recovery():
    w, h = train_mlr.train(samples=2048, classes=50, features=256, batch=256, iterations=50, lr=5.0, max_norm=0.05, fail_at=30, block=64)
    assert abs(h.loss[0] - math.log(50)) <= 1e-5, "all-zero weights: every class is equally likely"
    assert h.loss[-1] < 0.7 * h.loss[0] and all(math.isfinite(v) for v in h.loss + h.grad_norm)
    assert 0 < h.perturbation <= h.perturbation_bound and h.lost_blocks == 50
    assert h.saved_blocks == 25 * 50 and h.launches > 0
    assert bool(w.isfinite().all())


def test_steps_are_those_of_the_definition():
    """Ten clipped steps without a failure against the same loop in 64 bits.  A step's gradient is within 2^-18 of its
    norm (float32 sums), its factor likewise; steps of length lr * max_norm at most, so the weights are within
    10 * lr * max_norm * 2^-16 (an error of the weights changes the next gradient by less than itself here)."""
    kw = dict(samples=512, classes=20, features=64, batch=128, iterations=10, lr=1.0, max_norm=0.1, block=64)
    w, h = train_mlr.train(fail_at=0, **kw)
    x, y = train_mlr.make_data(512, 20, 64, 0)
    x, v = x.double(), torch.zeros(20, 64, dtype=torch.float64, device="cuda")
    order = torch.Generator(device="cuda").manual_seed(1)
    for it in range(10):
        at = torch.randint(0, 512, (128,), device="cuda", generator=order)
        z = x[at] @ v.T
        p = torch.softmax(z, 1)
        assert abs(h.loss[it] - float(torch.nn.functional.cross_entropy(z, y[at]))) <= 1e-4
        p[torch.arange(128), y[at]] -= 1
        g = p.T @ x[at] / 128
        n = float(g.norm())
        assert abs(h.grad_norm[it] - n) <= 1e-4 * n
        v -= g * min(1.0, 0.1 / n)
    assert float((w.double() - v).norm()) <= 10 * 0.1 * 2.0 ** -16


def test_command_line(capsys):
    train_mlr.main(["--samples", "256", "--classes", "10", "--features", "64", "--batch", "64", "--iterations", "8", "--fail-at", "5"])
    out = capsys.readouterr().out
    assert '"loss_last"' in out and '"perturbation"' in out
