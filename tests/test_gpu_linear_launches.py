"""Which way gradients go whose rows lie off 16-byte boundaries."""

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import LinearLayer, api  # noqa: E402

pytestmark = pytest.mark.gpu


def test_split_sums_of_float32_stay_split_where_rows_lie_anywhere():
    """Two split products and their joins after the copies' and dz's kernels.  Each result within 2^-18 of its norm, as the layer's own tests have it."""
    T, K, N = 2000, 301, 2000
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda") for s in ((T, K), (N, K), (T, N)))
    layer = LinearLayer(T, K, N, torch.float32, activation="gelu")
    _, slope = layer.forward_train(x, w)
    before = api.scar_linear_launch_count(layer.op)
    dx, dw, _ = layer.backward(dy, x, w, slope)
    assert api.scar_linear_launch_count(layer.op) - before == 6
    z = x.double() @ w.double().T
    dz = dy.double() * (0.5 * torch.special.erfc(-z / 2 ** 0.5) + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5)
    for got, want in ((dx, dz @ w.double()), (dw, dz.T @ x.double())):
        assert float((got.double() - want).norm()) <= 2.0 ** -18 * float(want.norm())
    layer.close()
