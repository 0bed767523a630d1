"""The linear layer's float32 as a whole: how far results are off in the norm, where single values' bounds are too wide to tell."""

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import LinearLayer  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,N", [(4096, 2048), (16384, 1000)])
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9, 16, 17, 32, 33, 100])
def test_long_sums_keep_their_precision_whatever_the_rows(rows, positive, pad, K, N):
    """At most 64 values of k meet in one accumulator of the matrix instructions, in four steps that may each cut up to 2^-23 of it: 2^-21.
    The up to 256 sums of those are added in registers, where roundings (2^-24 of a sum that grows to the whole, a third of it in the mean
    square, either way) come to less than sqrt(256) / 3 of 2^-24: 2^-21.  Sums of products with either sign are larger on their way than at
    their end by sqrt(K) / K of the sizes at most: no more than that in the norm.  What planes leave out is below 2^-22.  Together below 2^-20."""
    g = torch.Generator(device="cuda").manual_seed(rows + K)
    x, w = (torch.randn(n, K + pad, generator=g, device="cuda")[:, pad:] for n in (rows, N))
    if positive:
        x, w = x.abs_(), w.abs_()
    layer = LinearLayer(rows, K, N, torch.float32, activation="identity", forward_only=True)
    y, want = layer.forward(x, w), x.double() @ w.double().T
    assert float((y.double() - want).norm()) <= 2.0 ** -20 * float(want.norm())
    layer.close()
