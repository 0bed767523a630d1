"""Hidden layers beside a checkpoint: nothing is saved after a wait that gave up."""

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import ScarError, api, train_mlr  # noqa: E402
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
