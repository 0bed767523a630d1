"""The operators of a hidden layer together, as a network uses them: gradients of a whole step against automatic differentiation
in 64 bits and against differences, a captured step, the training loop with saves and a recovery."""

import math

import pytest

torch = pytest.importorskip("torch")

from hidden import mask  # noqa: E402
from paper_1810_07354_b200 import Dropout, LinearCrossEntropy, LinearLayer, ResidualNorm, train_mlr  # noqa: E402
from paper_1810_07354_b200.hidden import HiddenLayers  # noqa: E402

pytestmark = pytest.mark.gpu


def plain(net, p, x, step, dropout, seed):
    """The network in the parameters' type."""
    def norm(v, w):
        return v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * w

    def m(cols, which):
        return 1.0 if not dropout else torch.from_numpy(mask(net.batch, cols, dropout, seed, step * (net.blocks + 1) + which)).cuda()

    gelu = torch.nn.functional.gelu
    h = gelu(x @ p["w_in"].T + p["b_in"]) * m(net.hidden, 0)
    n = norm(h, p["pre0"])
    for i in range(net.blocks):
        a = gelu(n @ p[f"w1_{i}"].T + p[f"b1_{i}"])
        a = a * m(a.shape[1], i + 1)
        h = h + net.scale * p[f"gate{i}"] * norm(a @ p[f"w2_{i}"].T + p[f"b2_{i}"], p[f"post{i}"])
        n = norm(h, p[f"pre{i + 1}"])
    return n


@pytest.mark.parametrize("features,hidden,blocks,batch,dropout", [(40, 24, 1, 16, 0.0), (100, 64, 2, 50, 0.2), (513, 130, 3, 77, 0.1), (256, 520, 1, 200, 0.5), (33, 8, 0, 5, 0.1)])
def test_gradients_of_a_step(features, hidden, blocks, batch, dropout):
    """Each operator's float32 results are within about 2^-18 of their norm (their own tests say how); through 3 blocks of five of them
    and the loss, forward and backward, a gradient stays within 40 such steps: 2^-12 of its norm."""
    classes, seed = 37, 11
    net = HiddenLayers(features, hidden, blocks, batch, dropout=dropout, scale=0.5, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(1)
    net.params.add_(torch.randn(net.params.shape, generator=g, device="cuda"), alpha=0.05)
    x = torch.randn(batch, features, generator=g, device="cuda")
    w, y = torch.randn(classes, hidden, generator=g, device="cuda"), torch.randint(0, classes, (batch,), generator=g, device="cuda")
    xent = LinearCrossEntropy(batch, classes, hidden, torch.float32)
    n = net.forward(x, 5)
    loss, _, dn, dw = xent.loss_and_grad(n, w, y)
    net.backward(dn, 5)
    p = {k: v.double().requires_grad_() for k, v in net.p.items()}
    w64 = w.double().requires_grad_()
    want = torch.nn.functional.cross_entropy(plain(net, p, x.double(), 5, dropout, seed) @ w64.T, y)
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 2.0 ** -16 * max(1.0, float(want.detach()))
    for k, v in list(p.items()) + [("w", w64)]:
        got = dw if k == "w" else net.g[k]
        assert float((got.double() - v.grad).norm()) <= 2.0 ** -12 * float(v.grad.norm()) + 1e-9, k
    # another step has other masks, and the first one again the same result
    again = net.forward(x, 6)
    assert dropout == 0 or not torch.equal(n, again)
    net.kept = []
    assert torch.equal(n, net.forward(x, 5))
    net.close()
    xent.close()


def test_the_loss_moves_as_the_gradient_says():
    """Central differences of the loss along the gradient itself: steps of 2^-7 of a unit direction leave a cubic term below 2 % of
    the slope here (the loss' third derivative along a unit direction is below ten times its first), its rounding (2^-20) below 1 %."""
    net = HiddenLayers(60, 48, 2, 32, dropout=0.1, seed=3)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = torch.randn(32, 60, generator=g, device="cuda"), torch.randn(10, 48, generator=g, device="cuda")
    y = torch.randint(0, 10, (32,), generator=g, device="cuda")
    xent = LinearCrossEntropy(32, 10, 48, torch.float32)
    _, _, dn, _ = xent.loss_and_grad(net.forward(x, 1), w, y)
    net.backward(dn, 1)
    grad = net.grads.clone()
    norm = float(grad.norm())
    ends = []
    for s in (2.0 ** -7, -(2.0 ** -7)):
        net.params.add_(grad, alpha=s / norm)
        ends.append(float(xent.loss(net.forward(x, 1), w, y)[0]))
        net.kept = []
        net.params.add_(grad, alpha=-s / norm)
    assert abs((ends[0] - ends[1]) * 2.0 ** 6 - norm) <= 0.03 * norm
    net.close()
    xent.close()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,D,M,kind", [(5, 64, 200, "rms"), (130, 264, 520, "layer"), (64, 1001, 77, "layer"), (3, 4104, 512, "rms")])
def test_a_block_of_every_type(dt, T, D, M, kind):
    """Norm, layer up with a mask, layer down, gated norm onto the residual: forward and backward against the same chain in 64 bits on
    the operators' own intermediate values, a step of the chain at a time (a rounding of each result to the type: u of its norm)."""
    g = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    x, w1, w2, b1, b2, dy, dn = r(T, D), r(M, D) / D ** 0.5, r(D, M) / M ** 0.5, r(M), r(D), r(T, D), r(T, D)
    gate, post, pre = r(T, D), r(D), r(D)
    norm, up, down = ResidualNorm(T, D, dt, kind=kind), LinearLayer(T, D, M, dt, "silu"), LinearLayer(T, M, D, dt, "identity")
    m = Dropout(0.3, 9).mask(2)
    _, n0 = norm.forward(x, w_pre=pre)
    a, slope = up.forward_train(n0, w1, b1, dropout=m)
    f = down.forward(a, w2, b2)
    kw = dict(scale=0.7, gate=gate, w_post=post, w_pre=pre)
    y, n1 = norm.forward(x, f, **kw)
    got = norm.backward(dy, dn, y, f, **kw)
    da, dw2, db2 = down.backward(got["df"], a, w2, None)
    dn0, dw1, db1 = up.backward(da, n0, w1, slope, dropout=m)
    last = norm.backward(got["dx"], dn0, x, w_pre=pre)
    d = lambda t: t.double().requires_grad_()  # noqa: E731

    def n_of(v, w):
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, (D,), w, None, 1e-6)
        return torch.nn.functional.rms_norm(v, (D,), w, 1e-6)

    u = max({torch.float32: 2.0 ** -18, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dt], 2.0 ** -18)

    def near(got, want, steps, what):
        assert float((got.double() - want).norm()) <= steps * u * float(want.norm()) + 1e-4 * u * want.numel() ** 0.5, what

    scale = torch.from_numpy(mask(T, M, 0.3, 9, 2)).cuda()
    xs, ws = d(x), d(pre)
    want = n_of(xs, ws)
    near(n0, want, 1, "first norm")
    near(last["dx"], torch.autograd.grad(want, xs, dn0.double(), retain_graph=True)[0] + got["dx"].double(), 1, "dx of the first norm")
    near(last["dw_pre"], torch.autograd.grad(want, ws, dn0.double())[0], 1, "weight of the first norm")
    ns, w1s, b1s = d(n0), d(w1), d(b1)
    want = torch.nn.functional.silu(ns @ w1s.T + b1s) * scale
    near(a, want, 1, "up")
    for v, t, k in zip((dn0, dw1, db1), torch.autograd.grad(want, (ns, w1s, b1s), da.double()), ("dn0", "dw1", "db1")):
        near(v, t, 1, k)
    as_, w2s, b2s = d(a), d(w2), d(b2)
    want = as_ @ w2s.T + b2s
    near(f, want, 1, "down")
    for v, t, k in zip((da, dw2, db2), torch.autograd.grad(want, (as_, w2s, b2s), got["df"].double()), ("da", "dw2", "db2")):
        near(v, t, 1, k)
    xs, fs, gs, ps, qs = d(x), d(f), d(gate), d(post), d(pre)
    want = xs + 0.7 * gs * n_of(fs, ps)
    near(y, want, 1, "y")
    kept = want + (y.double() - want.detach())
    want_n = n_of(kept, qs)
    near(n1, want_n, 1, "n")
    for k, t in zip(("dx", "df", "dgate", "dw_post", "dw_pre"), torch.autograd.grad((want, want_n), (xs, fs, gs, ps, qs), (dy.double(), dn.double()))):
        near(got[k], t, 1, k)
    for op in (norm, up, down):
        op.close()


def test_training_with_hidden_layers_saves_and_a_recovery():
    kw = dict(samples=1024, classes=30, features=128, batch=128, iterations=30, lr=2.0, max_norm=0.05, fail_at=20, block=64, hidden=64, blocks=2, dropout=0.1)
    w, h = train_mlr.train(**kw)
    assert len(h.loss) == 30 and all(math.isfinite(v) for v in h.loss + h.grad_norm) and bool(w.isfinite().all())
    assert abs(h.loss[0] - math.log(30)) <= 1e-5, "the regression's weights begin at zero: every class is equally likely"
    assert 0 < h.perturbation <= h.perturbation_bound and h.saved_blocks > 0 and h.launches > 0
    again, h2 = train_mlr.train(**kw)
    assert torch.equal(w, again) and h.loss == h2.loss, "masks come from the seed and the step: a run repeats bit for bit"


def test_command_line_with_hidden_layers(capsys):
    train_mlr.main(["--samples", "256", "--classes", "10", "--features", "64", "--batch", "64", "--iterations", "8", "--fail-at", "5", "--hidden", "32", "--blocks", "1", "--dropout", "0.2"])
    out = capsys.readouterr().out
    assert '"loss_last"' in out and '"perturbation"' in out
