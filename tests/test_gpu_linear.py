"""The linear layer and its gradients against the definition in 64 bits.

Tolerances, derived from the formats and the lengths of the sums:

* a product's sum over K terms joins at most K/16 + 16 times, each join off by at most one unit: ``gamma(K) = (K/16 + 16) 2^-23``
  of the sum of absolute products; z is off by ``ez`` of that and a rounding of the bias' addition;
* activations move by at most 1.13 ez, their derivatives by 0.8 ez (relu: by 1 where |z| <= ez); evaluating them costs 2^-20 (the
  distribution function's formula 2^-22.6, float32 operations the rest), times 1 + |z|;
* the derivative is kept in float16 beside bfloat16 (2^-11, smallest half step 2^-25), else in float32;
* dz is rounded once to the operands' type (float32: 2^-23 for three planes), every result once.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from hidden import close, mask, smallest, unit  # noqa: E402
from paper_1810_07354_b200 import Dropout, LinearLayer, ScarError, api  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def gamma(k):
    return (k / 16 + 16) * 2.0 ** -23


def activation(z, act):
    if act == "identity":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    cdf = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5


def make(T, K, N, dt, seed=0, pad=0, bias=True, residual=True):
    g = torch.Generator(device="cuda").manual_seed(seed + T + K + N)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w = r(T, K + pad)[:, pad:].to(dt) if not pad else r(T, K + pad).to(dt)[:, pad:], (r(N, K + pad) * 1.5 / K ** 0.5).to(dt)[:, pad:]
    return x, w, r(N).to(dt) if bias else None, r(T, N + pad).to(dt)[:, pad:] if residual else None, r(T, N + pad).to(dt)[:, pad:]


def reference(x, w, b, res, dy, act, m):
    dt = x.dtype
    u, tiny = unit(dt), smallest(dt)
    f32, half_slope = dt == torch.float32, dt == torch.bfloat16
    x, w, dy = x.double(), w.double(), dy.double()
    K, N, T = x.shape[1], w.shape[0], x.shape[0]
    z = x @ w.T
    ez = gamma(K) * (x.abs() @ w.abs().T)
    if b is not None:
        z = z + b.double()
        ez = ez + 2.0 ** -23 * z.abs()
    a, s = activation(z, act)
    plain = act in ("identity", "relu")
    e_a = 1.13 * ez + (0 if plain else 2.0 ** -20 * z.abs() * (1 + ez))
    e_s = torch.zeros_like(z) if act == "identity" else (z.abs() <= ez).double() if act == "relu" else 0.8 * ez + 2.0 ** -20 * (1 + z.abs().clamp(max=8))
    if not plain:
        e_s = e_s + (2.0 ** -11 * s.abs() + 2.0 ** -25 if half_slope else 2.0 ** -24 * s.abs())
    y = m * a
    e_y = m * e_a + 2.0 ** -23 * y.abs()
    if res is not None:
        y = y + res.double()
        e_y = e_y + 2.0 ** -24 * y.abs()
    e_y = e_y + u * (y.abs() + e_y) + tiny
    dz = dy * m * s
    e_d = dy.abs() * m * e_s + 2.0 ** -22 * dz.abs()  # before dz is rounded
    e_dz = e_d + (2.0 ** -23 if f32 else u) * (dz.abs() + e_d) + tiny
    out = {"y": (y, e_y)}
    for k, p, q, e, n in (("dx", dz, w, e_dz, N), ("dw", dz.T, x, e_dz.T, T)):
        v = p @ q
        tol = e @ q.abs() + gamma(n) * (p.abs() @ q.abs())
        out[k] = v, tol + u * (v.abs() + tol) + tiny
    v, tol = dz.sum(0), e_d.sum(0) + (T / 8 + 64) * 2.0 ** -24 * dz.abs().sum(0)
    out["dbias"] = v, tol + u * (v.abs() + tol) + tiny
    return out


def check(layer, T, K, N, dt, act, p=0.0, **kw):
    x, w, b, res, dy = make(T, K, N, TYPES[dt], **kw)
    drop = Dropout(p, 31).mask(T) if p else None
    m = torch.from_numpy(mask(T, N, p, 31, T)).cuda() if p else torch.ones(T, N, dtype=torch.float64, device="cuda")
    want = reference(x, w, b, res, dy, act, m)
    y = layer.forward(x, w, bias=b, residual=res, dropout=drop)
    yt, slope = layer.forward_train(x, w, bias=b, residual=res, dropout=drop)
    dx, dw, db = layer.backward(dy, x, w, slope, dropout=drop)
    assert torch.equal(y, yt)
    layer.status()
    for k, got in (("y", y), ("dx", dx), ("dw", dw), ("dbias", db)):
        close(got, *want[k], f"{k} of {T} x {K} -> {N} {dt} {act}")
    # as a whole: two roundings (the derivative's is far below bfloat16's), each at most 3^-1/2 units in the mean square (values just above
    # a power of two, any fraction of a step equally likely): 0.82, and 1 with the few values of a small result; relu without a corner
    if T * K * N > 4096 and act != "relu":
        for k, got in (("dx", dx), ("dw", dw)):
            v = want[k][0]
            assert float((got.double() - v).norm()) <= max(unit(TYPES[dt]), 2.0 ** -19) * float(v.norm()) + 2 * smallest(TYPES[dt]) * v.numel() ** 0.5, k
    return x, w, b, res, dy, y, slope, dx, dw, db


SIZES = [(1, 1, 1), (1, 8, 8), (2, 3, 5), (7, 64, 64), (1, 300, 1000), (16, 1000, 33), (63, 65, 257), (64, 512, 512), (65, 100, 300), (129, 264, 72),
         (256, 256, 256), (257, 40, 1030), (300, 777, 129), (700, 8, 16), (2, 5000, 40), (40, 6000, 264), (3, 33, 9001), (1500, 128, 520)]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("act", ["identity", "relu", "gelu", "silu"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_every_output_is_within_its_bound(dt, act, T, K, N):
    layer = LinearLayer(T + 3, K, N, TYPES[dt], activation=act)
    check(layer, T, K, N, dt, act)
    check(layer, T, K, N, dt, act, p=0.3, bias=False, residual=False)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("T,K,N", [(5, 40, 72), (130, 264, 520), (70, 101, 203), (12, 512, 2048)])
def test_rows_of_wider_buffers(dt, pad, T, K, N):
    layer = LinearLayer(T, K, N, TYPES[dt], activation="gelu")
    check(layer, T, K, N, dt, "gelu", p=0.5, pad=pad)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 24, 31, 32, 33, 48, 64, 100])
def test_few_rows_of_a_wide_layer(dt, rows):
    layer = LinearLayer(100, 2056, 4104, TYPES[dt], activation="silu")
    check(layer, rows, 2056, 4104, dt, "silu", p=0.1)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_larger_sizes(dt):
    layer = LinearLayer(2000, 1024, 3000, TYPES[dt], activation="gelu")
    check(layer, 1900, 1024, 3000, dt, "gelu", p=0.1)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_results_repeat_and_rows_do_not_depend_on_one_another(dt):
    T, K, N = 200, 520, 1100
    layer = LinearLayer(T, K, N, TYPES[dt], activation="silu")
    x, w, b, res, dy = make(T, K, N, TYPES[dt])
    first = layer.forward_train(x, w, b, res) + layer.backward(dy, x, w, layer.forward_train(x, w, b, res)[1])
    for _ in range(10):
        again = layer.forward_train(x, w, b, res) + layer.backward(dy, x, w, first[1])
        assert all(torch.equal(p, q) for p, q in zip(first, again))
    x2, res2 = x.clone(), res.clone()
    x2[7], res2[9, 5] = float("nan"), float("inf")
    y = layer.forward(x2, w, b, res2)
    same = torch.ones(T, dtype=torch.bool, device="cuda")
    same[7] = same[9] = False
    assert torch.equal(y[same], first[0][same]) and bool(y[7].isnan().all()) and float(y[9, 5]) == float("inf")
    dy2 = dy.clone()
    dy2[3] = float("nan")
    dx, dw, db = layer.backward(dy2, x, w, first[1])
    same = torch.arange(T, device="cuda") != 3
    assert torch.equal(dx[same], first[2][same]) and bool(dx[3].isnan().all()) and bool(dw.isnan().all()) and bool(db.isnan().all())
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_far_values(dt, act):
    """Products far from 0 on both sides, where exponentials overflow and vanish; by a weight of one column."""
    v = torch.tensor([0.0, -0.0, 1e-8, 1e-3, 0.5, 1, 3, 6, 12, 40, 90, 300, 3e4], device="cuda")
    z = torch.cat([v, -v]).to(TYPES[dt])
    layer = LinearLayer(len(z), 1, 1, TYPES[dt], activation=act)
    one = torch.ones(1, 1, device="cuda", dtype=TYPES[dt])
    y, slope = layer.forward_train(z[:, None].contiguous(), one)
    a, s = activation(z.double(), act)
    assert bool(y.isfinite().all())
    u = unit(TYPES[dt])
    assert bool(((y[:, 0].double() - a).abs() <= u * a.abs() + 2.0 ** -20 * z.double().abs().clamp(max=8) + smallest(TYPES[dt])).all())
    assert bool(((slope[:, 0].double() - s).abs() <= 2.0 ** -11 * s.abs() + 2.0 ** -19).all())
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_no_rows_and_gradients_that_are_not_needed(dt):
    T, K, N = 33, 70, 90
    layer = LinearLayer(T, K, N, TYPES[dt], activation="gelu")
    x, w, b, res, dy = make(T, K, N, TYPES[dt])
    y, slope = layer.forward_train(x, w, b, res)
    dx, dw, db = layer.backward(dy, x, w, slope)
    for need in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = layer.backward(dy, x, w, slope, need_dx=need[0], need_dw=need[1], need_dbias=need[2])
        for n, g, full in zip(need, got, (dx, dw, db)):
            assert g is None if not n else float((g.double() - full.double()).norm()) <= 4 * max(unit(TYPES[dt]), 2.0 ** -20) * float(full.double().norm())
    y0, slope0 = layer.forward_train(x[:0], w, b, res[:0])
    dx0, dw0, db0 = layer.backward(dy[:0], x[:0], w, slope0, dw=torch.full_like(w, 5), dbias=torch.full_like(b, 5))
    assert y0.shape == (0, N) and dx0.shape == (0, K) and bool((dw0 == 0).all()) and bool((db0 == 0).all())
    with pytest.raises(ScarError) as e:
        layer.forward(torch.randn(T + 1, K, device="cuda").to(TYPES[dt]), w)
    assert e.value.code == -7
    layer.close()


def test_rows_behind_the_last_and_columns_between_rows_stay():
    T, K, N, dt = 37, 72, 136, torch.bfloat16
    layer = LinearLayer(64, K, N, dt, activation="gelu")
    x, w, b, res, dy = make(T, K, N, dt)
    y, dx, dw = (torch.full((n, c + 8), 7.0, device="cuda", dtype=dt) for n, c in ((T + 9, N), (T + 9, K), (N + 9, K)))
    slope = torch.full((T + 9, N), 7.0, device="cuda", dtype=torch.float16)
    layer.forward_train(x, w, b, res, out=y[:T, :N], slope=slope[:T])
    layer.backward(dy, x, w, slope[:T], dx=dx[:T, :K], dw=dw[:N, :K])
    for t, n, c in ((y, T, N), (dx, T, K), (dw, N, K)):
        assert bool((t[n:] == 7).all()) and bool((t[:, c:] == 7).all()) and not bool((t[:n, :c] == 7).all())
    assert bool((slope[T:] == 7).all())
    layer.close()


def test_the_residual_as_the_output():
    for dt in TYPES.values():
        for T, K, N in ((50, 80, 304), (50, 80, 303), (3, 2048, 512)):
            layer = LinearLayer(T, K, N, dt, activation="relu")
            x, w, b, res, _ = make(T, K, N, dt)
            want = layer.forward(x, w, b, res)
            assert layer.forward(x, w, b, res, out=res) is res and torch.equal(res, want)
            layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_captured_and_replayed(dt):
    """Forward and backward in one graph, replayed with other values and another mask; an eager call of the same operator between."""
    T, K, N = 96, 256, 384
    stream = torch.cuda.Stream()
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    layer, drop = LinearLayer(T, K, N, TYPES[dt], activation="gelu", stream=stream), Dropout(0.2, 5, stream=stream)
    x, w, b, res, dy = make(T, K, N, TYPES[dt])

    def step(at):
        y, slope = layer.forward_train(x, w, b, res, dropout=drop.mask(at))
        return (y, *layer.backward(dy, x, w, slope, dropout=drop.mask(at)))

    with torch.cuda.stream(stream):
        step(offset)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step(offset)
    for at in (1, 2):
        x.copy_(make(T, K, N, TYPES[dt], seed=at)[0])
        offset.fill_(at)
        torch.cuda.synchronize()
        want = step(at)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    del graph
    layer.close()


def test_differences():
    """The gradients of float32 against central differences along random directions: with steps of 2^-6 the cubic term is below 1e-4 of
    the sum of squares that bounds the slope, the rounding of the loss (2^-22 of the sum of its terms' sizes) below 1e-4 of the slope."""
    T, K, N = 40, 60, 80
    for act in ("identity", "gelu", "silu"):
        layer, drop = LinearLayer(T, K, N, torch.float32, activation=act), Dropout(0.25, 8).mask(3)
        x, w, b, res, dy = make(T, K, N, torch.float32, seed=1)
        _, slope = layer.forward_train(x, w, b, res, dropout=drop)
        grads = layer.backward(dy, x, w, slope, dropout=drop)
        for i, g in enumerate(grads):
            d = torch.randn_like(g)
            d /= d.norm()
            h, at = 2.0 ** -6, [x, w, b]
            loss = []
            for sign in (1, -1):
                moved = list(at)
                moved[i] = at[i] + sign * h * d
                loss.append(float((layer.forward(*moved, res, dropout=drop).double() * dy.double()).sum()))
            assert abs((loss[0] - loss[1]) / (2 * h) - float((g.double() * d.double()).sum())) <= 2e-3 * float(g.double().norm()), (act, i)
        layer.close()


def test_reports_of_a_wait_that_gave_up():
    layer = LinearLayer(8, 16, 16, torch.float32)
    x, w, b, res, _ = make(8, 16, 16, torch.float32)
    layer.forward(x, w)
    layer.status()
    api.scar_linear_selftest_arm_timeout(layer.op)
    layer.forward(x, w)
    with pytest.raises(ScarError) as e:
        layer.status()
    assert e.value.code == -6
    layer.status()
    layer.forward(x, w)
    layer.status()
    layer.close()


def test_far_rows():
    """Rows whose offsets pass 2^32 bytes and elements."""
    T, K, N, far = 3, 64, 128, (1 << 31) + 64
    buf = torch.empty(2 * far + K, dtype=torch.bfloat16, device="cuda")
    layer = LinearLayer(T, K, N, torch.bfloat16, activation="silu")
    x, w, b, res, dy = make(T, K, N, torch.bfloat16)
    wide = buf.as_strided((T, K), (far, 1))
    wide.copy_(x)
    assert torch.equal(layer.forward(wide, w, b, res), layer.forward(x, w, b, res))
    out = buf.as_strided((T, K), (far, 1))
    _, slope = layer.forward_train(x, w, b, res)
    dx = layer.backward(dy, x, w, slope)[0]
    layer.backward(dy, x, w, slope, dx=out)
    assert torch.equal(out, dx)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows", [1, 5, 9, 16, 17, 32])
@pytest.mark.parametrize("K,N,pad", [(7, 40, 0), (31, 65, 1), (257, 130, 0), (257, 130, 5), (1001, 36, 2), (1002, 300, 0), (1004, 7, 0), (3000, 33, 1)])
def test_few_rows_anywhere(dt, rows, K, N, pad):
    layer = LinearLayer(rows, K, N, TYPES[dt], activation="gelu")
    check(layer, rows, K, N, dt, "gelu", p=0.2, pad=pad)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("off,more", [(0, 1), (1, 2), (3, 8), (2, 4), (5, 3)])
@pytest.mark.parametrize("T,K,N", [(3, 40, 72), (20, 101, 33), (70, 130, 203), (300, 264, 520)])
def test_results_between_other_values(dt, off, more, T, K, N):
    """Outputs in the middle of wider rows, wherever these begin: what lies beside them stays, and the results are those of whole tensors."""
    t = TYPES[dt]
    layer = LinearLayer(T, K, N, t, activation="silu")
    x, w, b, res, dy = make(T, K, N, t)
    y, slope = layer.forward_train(x, w, b, res)
    dx, dw, _ = layer.backward(dy, x, w, slope)
    wide = [torch.full((n, off + c + more), 7.0, device="cuda", dtype=t) for n, c in ((T, N), (T, K), (N, K))]
    part = [v[:, off: off + c] for v, c in zip(wide, (N, K, K))]
    layer.forward(x, w, b, res, out=part[0])
    layer.backward(dy, x, w, slope, dx=part[1], dw=part[2])
    u = 4 * max(unit(t), 2.0 ** -20)  # sums may be split elsewhere: two roundings apart
    for v, p, whole, c in zip(wide, part, (y, dx, dw), (N, K, K)):
        assert float((p.double() - whole.double()).norm()) <= u * float(whole.double().norm())
        assert bool((v[:, :off] == 7).all()) and bool((v[:, off + c:] == 7).all())
    layer.close()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_many_rows_off_every_boundary(dt):
    """More than the parts' room holds: results and residual go the product's own way."""
    T, K, N = 4200, 40, 4101
    layer = LinearLayer(T, K, N, TYPES[dt], activation="gelu")
    check(layer, T, K, N, dt, "gelu", p=0.1, pad=1)
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_gradients_of_no_rows_of_a_single_output(dt):
    """A matrix of one row has no use for its pitch, whatever is given for it."""
    layer = LinearLayer(8, 37, 1, TYPES[dt], activation="identity")
    w = torch.ones(1, 37, device="cuda", dtype=TYPES[dt])
    dw, db = torch.full_like(w, 5), torch.full((1,), 5, device="cuda", dtype=TYPES[dt])
    api.scar_linear_backward(layer.op, None, 0, None, 0, w.data_ptr(), 0, None, None, 0, None, 0, dw.data_ptr(), 0, db.data_ptr())
    layer.status()
    assert bool((dw == 0).all()) and bool((db == 0).all())
    layer.close()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("act,pad", [("gelu", 0), ("silu", 3), ("identity", 8)])
@pytest.mark.parametrize("K,N", [(40, 17), (129, 64), (1000, 1001), (264, 20000)])
@pytest.mark.parametrize("T", [1, 2, 7, 16])
def test_few_rows_have_no_rounding_but_the_results_own(dt, act, pad, K, N, T):
    """Gradients against the 64-bit ones rounded to the type.  On top of that rounding (a share of up to 1 unit, 0.4 in the mean square at
    least) there is the derivative's (2^-11 beside bfloat16, 2^-24 beside float16) and dz's second part (2^-16 and 2^-22): below 2^-3 of it,
    which adds 2^-7 in the mean square; sums of up to 20000 values 2^-13 of a unit of bfloat16, and of float16 2^-12 of their absolute
    products' sum over 2^-11 of the result: 2^-1.  Together below 1.15 times."""
    layer = LinearLayer(40, K, N, TYPES[dt], activation=act)
    x, w, b, res, dy = make(T, K, N, TYPES[dt], pad=pad)
    drop = Dropout(0.25, 31).mask(T)
    m = torch.from_numpy(mask(T, N, 0.25, 31, T)).cuda()
    want = reference(x, w, b, res, dy, act, m)
    _, slope = layer.forward_train(x, w, bias=b, residual=res, dropout=drop)
    wide = [torch.zeros(n, K + pad, device="cuda", dtype=TYPES[dt])[:, pad:] for n in (T, N)]
    dx, dw, db = layer.backward(dy, x, w, slope, dropout=drop, dx=wide[0], dw=wide[1])
    for k, got in (("dx", dx), ("dw", dw)):
        v = want[k][0]
        once = float((v.to(TYPES[dt]).double() - v).norm())
        assert float((got.double() - v).norm()) <= 1.15 * once + 2 * smallest(TYPES[dt]) * v.numel() ** 0.5, k
    only = layer.backward(dy, x, w, slope, dropout=drop, need_dw=False)[0], layer.backward(dy, x, w, slope, dropout=drop, need_dx=False)[1]
    assert torch.equal(only[0], dx) and torch.equal(only[1], dw)
    layer.close()


def test_values_beyond_float16_of_few_rows_are_infinite():
    layer = LinearLayer(4, 8, 8, torch.float16, activation="identity")
    x, w = torch.eye(4, 8, device="cuda").half(), torch.eye(8, device="cuda").half()
    dy = torch.zeros(4, 8, device="cuda").half()
    dy[1, 2] = 60000.0
    for seed in range(8):  # where it is kept it is doubled: 120000
        drop = Dropout(0.5, seed).mask(0)
        kept = bool(mask(4, 8, 0.5, seed, 0)[1, 2])
        dx, dw, db = layer.backward(dy, x, w, None, dropout=drop)
        assert not bool(dx.isnan().any()) or kept
        assert (float(db[2]) == float("inf")) == kept
        if not kept:
            assert bool((dx == 0).all()) and bool((dw == 0).all())
        else:
            assert float(dx[1, 2]) == float("inf") and float(dw[2, 1]) == float("inf")
    layer.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,K,N", [(3, 129, 70), (16, 256, 1000)])
def test_few_rows_captured(dt, T, K, N):
    """Forward and backward in one graph, replayed on other inputs: the bits of the same calls made one by one."""
    stream = torch.cuda.Stream()
    layer = LinearLayer(16, K, N, TYPES[dt], activation="silu", stream=stream)
    x, w, b, res, dy = make(T, K, N, TYPES[dt])
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = Dropout(0.25, 5, stream=stream).mask(offset)

    def step():
        y, slope = layer.forward_train(x, w, bias=b, residual=res, dropout=drop)
        return (y, *layer.backward(dy, x, w, slope, dropout=drop))

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        for i in range(3):
            offset.fill_(i)
            dy.mul_(-0.5)
            x.add_(0.25)
            graph.replay()
            want = step()
            stream.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(got, want))
    layer.status()
    layer.close()
