"""The linear layer's float32 as a whole: how far results are off in the norm, where single values' bounds are too wide to tell."""

import pytest

torch = pytest.importorskip("torch")

import math  # noqa: E402

from paper_1810_07354_b200 import Dropout, LinearLayer  # noqa: E402

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


@pytest.mark.parametrize("rows", [1, 4, 20, 4096])
def test_gelu_and_its_derivative_to_a_few_units(rows):
    """z comes as the bias of a product of zeros, so nothing but the activation is rounded.  The exponential's instruction is off by 2^-22, the
    reciprocal's by 2^-23, a polynomial's last steps by 2^-22 and three products by 2^-24 each: below 2^-20 of the value, of the
    derivative 2^-20 of its two terms' sizes.  From -9 on: below -13 results leave float32's ordinary range."""
    n = 40960 // rows
    z = torch.linspace(-9.0, 9.0, 40960, device="cuda").view(n, rows).t().contiguous() if rows > 1 else torch.linspace(-9.0, 9.0, n, device="cuda")[None]
    # one column of x for each output: z = x w^T + bias with x = 1, w = 0 has the bias for z
    layer = LinearLayer(rows, 1, n, torch.float32, activation="gelu")
    for r in sorted({0, rows // 2, rows - 1}):
        bias = z[r].contiguous()
        y, slope = layer.forward_train(torch.ones(rows, 1, device="cuda"), torch.zeros(n, 1, device="cuda"), bias=bias)
        b = bias.double()
        cdf, part = 0.5 * torch.special.erfc(-b / 2 ** 0.5), b * torch.exp(-b * b / 2) / (2 * math.pi) ** 0.5
        assert float(((y[r].double() - b * cdf).abs() / (b * cdf).abs().clamp(min=1e-300)).max()) <= 2.0 ** -20
        assert float(((slope[r, :n].double() - cdf - part).abs() / (cdf + part.abs())).max()) <= 2.0 ** -20
    layer.close()


def test_gelu_of_values_at_the_ends_of_the_range():
    z = torch.tensor([float("nan"), float("inf"), 3e38, 1e20, 40.0, 0.0, -40.0, -1e20, -3e38], device="cuda")
    layer = LinearLayer(1, 1, 9, torch.float32, activation="gelu")
    y, slope = layer.forward_train(torch.ones(1, 1, device="cuda"), torch.zeros(9, 1, device="cuda"), bias=z)
    assert bool(y[0, 0].isnan()) and bool(slope[0, 0].isnan())
    assert torch.equal(y[0, 1:], z[1:].clamp(min=0)) and torch.equal(slope[0, 2:9], torch.tensor([1, 1, 1, 0.5, 0, 0, 0], device="cuda"))
    layer.close()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,K,N,most", [(17, 300, 1, 1.15), (17, 129, 64, 1.15), (64, 1000, 8, 1.15), (100, 264, 7, 1.15), (512, 40, 4, 1.15), (2000, 65, 1, 1.15),
                                        (33, 4096, 62, 1.15), (17, 300, 130, 2.24), (300, 300, 8, 2.24), (1030, 100, 2, 2.24), (2100, 300, 1, 2.24)])
def test_gradients_of_few_values_have_no_rounding_but_the_results_own(dt, T, K, N, most):
    """dx and dw beside the 64-bit ones rounded to the type.  dz in two values is off by 2^-16 (bfloat16) or 2^-22 of itself, the derivative beside
    bfloat16 by 2^-11, sums of up to 2048 products by 2^-13 of a unit: well below the 1.15 times.  dz rounded once adds an error
    as large as the result's rounding where both have many values anywhere in their binades (1.41 times together).  Proof of 2.24 for any: a
    rounding takes up to half a step, u 2^e in [2^e, 2^(e + 1)), so its mean square lies between u^2 / 12 (values just below
    2^(e + 1)) and u^2 / 3 (just above 2^e) of the values'; products with rows of independent signs keep that share, so the two are
    at most 4 : 1 in the mean square: (1 + 4)^1/2."""
    g = torch.Generator(device="cuda").manual_seed(T + N)
    drop = Dropout(0.25, 3).mask(7)
    layer = LinearLayer(T, K, N, dt, activation="silu")
    ones = LinearLayer(T, K, N, dt, activation="identity")
    for _ in range(6):
        x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(dt) for s in ((T, K), (N, K), (T, N)))
        w.div_(K ** 0.5)
        keep = ones.forward(torch.zeros_like(x), w, bias=torch.ones(N, device="cuda", dtype=dt), dropout=drop) != 0
        _, slope = layer.forward_train(x, w, dropout=drop)
        dx, dw, _ = layer.backward(dy, x, w, slope, dropout=drop)
        z = x.double() @ w.double().T
        s = torch.sigmoid(z)
        dz = dy.double() * keep / 0.75 * s * (1 + z * (1 - s))
        for got, want in ((dx, dz @ w.double()), (dw, dz.T @ x.double())):
            once = float((want.to(dt).double() - want).norm())
            assert float((got.double() - want).norm()) <= most * once
    layer.close()
    ones.close()


@pytest.mark.parametrize("T,N", [(4, 8), (40, 64)])
def test_a_float16_value_of_dz_beyond_the_range_is_infinite_in_its_row_and_column_alone(T, N):
    """dy = 60000 where it is kept and doubled; dz in two values and in one.  An infinity times a weight of 0 is a NaN, times others it keeps
    its sign; everything else is what it is without that value."""
    K = 8
    layer = LinearLayer(T, K, N, torch.float16, activation="identity")
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.randn(T, K, generator=g, device="cuda").half(), torch.randn(N, K, generator=g, device="cuda").half()
    w[2, 5], x[1, 3] = 0, 0
    dy = torch.randn(T, N, generator=g, device="cuda").half()
    ones = torch.ones(N, device="cuda").half()
    for seed in range(6):
        drop = Dropout(0.5, seed).mask(0)
        if float(layer.forward(torch.zeros_like(x), w, bias=ones, dropout=drop)[1, 2]) == 0:
            continue
        dy[1, 2] = 0.0
        dx0, dw0, db0 = (v.clone() for v in layer.backward(dy, x, w, None, dropout=drop))
        dy[1, 2] = 60000.0
        dx, dw, db = layer.backward(dy, x, w, None, dropout=drop)
        for got, base, line, other in ((dx, dx0, 1, w[2]), (dw, dw0, 2, x[1])):
            want = base.clone()
            want[line] = other.float().sign() * float("inf")  # NaN where the other factor is 0
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=1.0), want.nan_to_num(nan=1.0))
        want = db0.clone()
        want[2] = float("inf")
        assert torch.equal(db, want)
    layer.close()
