"""The norms' own way out of a wait that gave up: the call ends by itself, says so, and the operator is as good as before.

A warp of the first CTA takes its first wait as one that ran out (the library's hook), so the waits that depend on it run into their
two seconds each, those for rows and those for sums one after the other at most.  Rows cut over the CTAs of a cluster are what this is
about: one CTA is through long before the others."""

import time

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import ResidualNorm, ScarError, api  # noqa: E402

pytestmark = pytest.mark.gpu


def results(op, kind, x, f, dy, dn, gate):
    kw = dict(scale=0.5, gate=gate, rows_per_gate=3)
    if kind == "layer":
        kw["b_post"] = torch.ones_like(x[0]).contiguous()
    kw["w_pre"] = torch.full_like(x[0], 0.5).contiguous()
    y, n = op.forward(x, f, **kw)
    return y, n, lambda: op.backward(dy, dn, y, f, **kw), lambda: op.forward(x, f, **kw)


@pytest.mark.parametrize("dt,kind,T,D,warp", [
    (torch.bfloat16, "rms", 40, 64, 1),       # a single warp
    (torch.float32, "layer", 3000, 1001, 1),  # rows anywhere, a CTA a row
    (torch.bfloat16, "rms", 2000, 5000, 1),   # two CTAs a row
    (torch.bfloat16, "layer", 2000, 8200, 3),
    (torch.float16, "rms", 1500, 8195, 2),    # rows anywhere, three of them
    (torch.float32, "layer", 700, 16384, 1),  # four
    (torch.float32, "rms", 700, 16384, 100),
])
def test_a_call_whose_wait_gave_up_ends_and_says_so(dt, kind, T, D, warp):
    op = ResidualNorm(T, D, dt, kind=kind)
    g = torch.Generator(device="cuda").manual_seed(T + D)
    x, f, dy, dn = (torch.randn(T, D, generator=g, device="cuda").to(dt) for _ in range(4))
    gate = torch.randn(-(-T // 3), D, generator=g, device="cuda").to(dt)
    y, n, backward, forward = results(op, kind, x, f, dy, dn, gate)
    grads = backward()
    op.status()
    for call in (forward, backward):
        for _ in range(warp):
            api.scar_resnorm_selftest_arm_timeout(op.op)
        at = time.monotonic()
        call()
        with pytest.raises(ScarError) as e:
            op.status()
        assert e.value.code == -6 and time.monotonic() - at < 30
        op.status()
        again, after = forward(), backward()
        op.status()
        assert torch.equal(again[0], y) and torch.equal(again[1], n)
        assert all(v is None or torch.equal(v, after[k]) for k, v in grads.items())
    op.close()
