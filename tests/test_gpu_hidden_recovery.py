"""Hidden layers beside a checkpoint: steps taken again after a recovery are the same steps, and nothing is saved after a wait that gave up."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import GradientNorm, LinearCrossEntropy, ScarCheckpoint, ScarError, api, train_mlr  # noqa: E402
from paper_1810_07354_b200.hidden import HiddenLayers  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["first", "down", "norm"])
def test_training_stops_before_it_saves_what_a_kernel_did_not_finish(monkeypatch, which):
    forward, saves = HiddenLayers.forward, []

    def failing(self, x, step):
        if step == 5:
            arm = api.scar_resnorm_selftest_arm_timeout if which == "norm" else api.scar_linear_selftest_arm_timeout
            arm(getattr(self, which).op)
        return forward(self, x, step)

    save = api.ScarCheckpoint.priority_save_k
    monkeypatch.setattr(HiddenLayers, "forward", failing)
    monkeypatch.setattr(api.ScarCheckpoint, "priority_save_k", lambda self, k, sync=True: saves.append(k) or save(self, k, sync))
    kw = dict(samples=256, classes=10, features=64, batch=64, lr=1.0, max_norm=0.05, fail_at=100, block=64, hidden=32, blocks=1, dropout=0.1)
    with pytest.raises(ScarError) as e:
        train_mlr.train(iterations=20, **kw)  # saves after every second step
    assert e.value.code == -6 and len(saves) == 2
    with pytest.raises(ScarError):
        train_mlr.train(iterations=5, **kw)  # and not without a word where the last step is the one


def test_steps_taken_again_after_a_recovery_have_the_same_masks():
    """All parameters are lost two steps after they were saved whole, and come back; the two steps are taken again with their own numbers
    and give the same parameters bit for bit, and another mask (another number) does not."""
    batch, features, hidden, classes = 96, 72, 40, 11
    net = HiddenLayers(features, hidden, 2, batch, dropout=0.3, seed=5)
    at = net.params.numel()
    params, grads = torch.zeros(at + classes * hidden, device="cuda"), torch.zeros(at + classes * hidden, device="cuda")
    params[:at] = net.params
    params[at:].normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    net.place(params[:at], grads[:at])
    w, dw = params[at:].view(classes, hidden), grads[at:].view(classes, hidden)
    xent, clip, ck = LinearCrossEntropy(batch, classes, hidden, torch.float32), GradientNorm([grads]), ScarCheckpoint(params, n_shards=4, block_elems=64)

    def step(number, masks=None):
        g = torch.Generator(device="cuda").manual_seed(100 + number)  # the step's rows
        x, y = torch.randn(batch, features, generator=g, device="cuda"), torch.randint(0, classes, (batch,), generator=g, device="cuda")
        n = net.forward(x, number if masks is None else masks)
        kept = [k[2] != 0 for k in net.kept]  # what the masks left of h and of every block's inner layer
        _, _, dn, _ = xent.loss_and_grad(n, w, y, dw=dw)
        net.backward(dn, number if masks is None else masks)
        clip.clip(1.0)
        params.sub_(grads, alpha=0.5)
        return kept

    step(1)
    step(2)
    assert int(ck.priority_save_k(ck.n_blocks).k) == ck.n_blocks
    saved = params.clone()
    masks = step(3) + step(4)
    reached = params.clone()
    params.fill_(float("nan"))
    ck.recover_partial(np.ones(4, dtype=np.uint8))
    assert torch.equal(params, saved) and not torch.equal(saved, reached)
    again = step(3) + step(4)
    assert all(torch.equal(a, b) for a, b in zip(masks, again)) and torch.equal(params, reached)
    assert all(0.2 < 1 - float(m.double().mean()) < 0.4 for m in masks)
    params.copy_(saved)
    other = step(3, masks=30) + step(4, masks=40)
    assert not any(torch.equal(a, b) for a, b in zip(masks, other)) and not torch.equal(params, reached)
    for op in (net, xent, clip, ck):
        op.close()
