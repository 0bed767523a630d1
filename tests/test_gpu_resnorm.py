"""The norms around a residual block and their gradients against the definition in 64 bits.

Tolerances: sums over a row are trees over runs of at most 32 values (at most 64 joins of 2^-24 each), and at most four of such sums
and 16 single operations lie between an input and a result: 2^-17 of the sum of the sizes of the terms that make a result.  Sums over
T rows join at most T + 64 times.  Every result is rounded once.  A row's mean may be off by 2^-21 of its largest value, which moves
the normalised values by that over the deviation."""

import pytest

torch = pytest.importorskip("torch")

from hidden import close, smallest, unit  # noqa: E402
from paper_1810_07354_b200 import ResidualNorm, ScarError  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
LOSS = 2.0 ** -17


def normed(v, layer):
    """Normalised rows, 1 / deviation, and what the normalised values may be off by."""
    m = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    r = ((v - m).square().mean(1, keepdim=True) + EPS).rsqrt()
    hat = (v - m) * r
    off = LOSS * hat.abs() + (2.0 ** -21 * v.abs().amax(1, keepdim=True) * r if layer else 0)
    return hat, r, off


def norm_back(h, hat, off, r, layer, e_h):
    """The gradient through a norm, and its bound; e_h: of h."""
    mh = h.mean(1, keepdim=True) if layer else 0
    mhh = (h * hat).mean(1, keepdim=True)
    got = r * (h - mh - hat * mhh)
    size = h.abs() + (h.abs().mean(1, keepdim=True) if layer else 0) + hat.abs() * (h * hat).abs().mean(1, keepdim=True)
    e_mhh = (e_h * hat.abs() + h.abs() * off).mean(1, keepdim=True)
    tol = r * (e_h + (e_h.mean(1, keepdim=True) if layer else 0) + off * mhh.abs() + hat.abs() * e_mhh) + LOSS * r * size
    return got, tol


class Case:
    def __init__(self, T, D, dt, kind="rms", post=True, pre=True, group=0, pad=0, weights=True, seed=0, mean=0.3):
        g = torch.Generator(device="cuda").manual_seed(seed + T + D)
        dtype = TYPES[dt]

        def r(n, d, spread=1.0, at=0.0, pad=pad):
            return (torch.randn(n, d + pad, generator=g, device="cuda") * spread + at).to(dtype)[:, pad:]

        def vec(at):
            return (torch.randn(D, generator=g, device="cuda") * 0.2 + at).to(dtype) if weights else None

        self.kind, self.layer, self.post, self.pre, self.group, self.dtype = kind, kind == "layer", post, pre, group, dtype
        self.x, self.f, self.dy, self.dn = r(T, D, 2.0, mean), r(T, D, 0.5, mean), r(T, D), r(T, D) if pre else None
        self.gate = r(-(-T // group), D, 0.3, 0.5) if group else None
        self.kw = dict(post=post, pre=pre, scale=0.7, gate=self.gate, rows_per_gate=group or 1, w_post=vec(1) if post else None, w_pre=vec(1) if pre else None,
                       b_post=vec(0) if post and self.layer else None, b_pre=vec(0) if pre and self.layer else None)

    def d(self, name):
        v = self.kw[name]
        return torch.as_tensor(1.0 if name[0] == "w" else 0.0, dtype=torch.float64, device="cuda") if v is None else v.double()

    def check(self, op):
        T, D = self.x.shape
        u, tiny, kw = unit(self.dtype), smallest(self.dtype), self.kw
        done = lambda v, e: (v, e + u * (v.abs() + e) + tiny)  # noqa: E731
        y, n = op.forward(self.x, self.f, **kw)
        x, f = self.x.double(), self.f.double()
        scale = torch.tensor(kw["scale"], dtype=torch.float32).double().item()
        each = torch.arange(T, device="cuda") // (self.group or 1)
        gate = torch.ones_like(x) if self.gate is None else self.gate.double()[each]
        hat, r, off = normed(f, self.layer) if self.post else (f, None, torch.zeros_like(f))
        w, b = self.d("w_post"), self.d("b_post")
        u_, e_u = hat * w + b, off * w.abs() + 2.0 ** -23 * ((hat * w).abs() + b.abs())
        want = x + scale * gate * u_
        close(y, *done(want, scale * gate.abs() * e_u + 2.0 ** -22 * (x.abs() + (scale * gate * u_).abs())), "y")
        if self.pre:
            yhat, yr, yoff = normed(y.double(), self.layer)  # of the values handed on
            w2, b2 = self.d("w_pre"), self.d("b_pre")
            close(n, *done(yhat * w2 + b2, yoff * w2.abs() + 2.0 ** -23 * ((yhat * w2).abs() + b2.abs())), "n")
        got = op.backward(self.dy, self.dn, y, self.f, **kw)
        dY, e = self.dy.double(), torch.zeros_like(x)
        rows = lambda t, tol: (t.sum(0), tol.sum(0) + (T + 64) * 2.0 ** -24 * t.abs().sum(0))  # noqa: E731
        if self.pre:
            dn = self.dn.double()
            back, e = norm_back(dn * w2, yhat, yoff, yr, self.layer, 2.0 ** -24 * (dn * w2).abs())
            dY, e = dY + back, e + 2.0 ** -23 * (dY.abs() + back.abs())
            if kw["w_pre"] is not None:
                close(got["dw_pre"], *done(*rows(dn * yhat, dn.abs() * yoff)), "dw_pre")
            if kw["b_pre"] is not None:
                close(got["db_pre"], *done(*rows(dn, torch.zeros_like(dn))), "db_pre")
        close(got["dx"], *done(dY, e), "dx")
        if self.gate is not None:
            t, tol = scale * dY * u_, scale * (e * u_.abs() + dY.abs() * e_u) + 2.0 ** -22 * (scale * dY * u_).abs()
            zero = torch.zeros_like(self.gate.double())
            total = zero.index_add(0, each, t)
            close(got["dgate"], *done(total, zero.index_add(0, each, tol) + (min(T, self.group) + 64) * 2.0 ** -24 * zero.index_add(0, each, t.abs())), "dgate")
        du, e_du = scale * gate * dY, scale * gate.abs() * e + 2.0 ** -22 * (scale * gate * dY).abs()
        if self.post:
            if kw["w_post"] is not None:
                close(got["dw_post"], *done(*rows(du * hat, e_du * hat.abs() + du.abs() * off)), "dw_post")
            if kw["b_post"] is not None:
                close(got["db_post"], *done(*rows(du, e_du)), "db_post")
            du, e_du = norm_back(du * w, hat, off, r, self.layer, e_du * w.abs() + 2.0 ** -24 * (du * w).abs())
        close(got["df"], *done(du, e_du), "df")
        assert {k for k, v in got.items() if v is None} == {k for k, v in (("dgate", self.gate), *((f"d{n}", kw[n]) for n in ("w_post", "b_post", "w_pre", "b_pre"))) if v is None}
        return y, n, got


SIZES = [(1, 1), (1, 8), (3, 5), (2, 256), (7, 257), (33, 64), (130, 100), (64, 1000), (300, 24), (5, 4096), (4, 4097), (9, 5000), (3, 8192), (2, 8200), (3, 16384),
         (2, 16383), (1000, 520), (700, 1537), (160, 3500)]


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,D", SIZES)
def test_every_output_is_within_its_bound(dt, kind, T, D):
    op = ResidualNorm(T + 2, D, TYPES[dt], kind=kind, eps=EPS)
    Case(T, D, dt, kind).check(op)
    Case(T, D, dt, kind, group=1, weights=False).check(op)
    Case(T, D, dt, kind, group=T, pad=3).check(op)
    Case(T, D, dt, kind, group=max(1, T // 3), pad=8).check(op)
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("group", [0, 1, 7, 5000])
def test_blocks_without_one_norm_or_both(dt, kind, post, pre, group):
    for T, D in ((50, 130), (400, 1024)):
        op = ResidualNorm(T, D, TYPES[dt], kind=kind, eps=EPS)
        Case(T, D, dt, kind, post, pre, min(group, T)).check(op)
        op.close()


@pytest.mark.parametrize("group", [2, 3, 10, 64, 333, 1000, 1999])
def test_gates_that_end_anywhere(group):
    T, D = 2000, 264
    op = ResidualNorm(T, D, torch.float32, kind="layer", eps=EPS)
    Case(T, D, "f32", "layer", group=group).check(op)
    Case(T - 1, D, "f32", "layer", group=group).check(op)
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
def test_rows_far_from_zero_keep_their_deviation(dt):
    """A mean of 40 deviations and more: the statistics are taken around the mean."""
    op = ResidualNorm(64, 1000, TYPES[dt], kind="layer", eps=EPS)
    Case(64, 1000, dt, "layer", mean=40.0 if dt == "f32" else 8.0).check(op)
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_the_norm_alone(dt, kind):
    """Without a block: the first norm of a model, its input the output."""
    T, D = 70, 520
    c = Case(T, D, dt, kind)
    op = ResidualNorm(T, D, TYPES[dt], kind=kind, eps=EPS)
    kw = dict(w_pre=c.kw["w_pre"], b_pre=c.kw["b_pre"])
    y, n = op.forward(c.x, **kw)
    assert y is c.x
    copy = torch.empty_like(c.x)
    y2, n2 = op.forward(c.x, y=copy, **kw)
    assert y2 is copy and torch.equal(copy, c.x) and torch.equal(n, n2)
    want = Case(T, D, dt, kind, post=False)
    zero = torch.zeros_like(c.f)
    got = op.backward(c.dy, c.dn, c.x, **kw)
    full = op.backward(c.dy, c.dn, c.x, zero, post=False, **kw)
    assert all(torch.equal(got[k], full[k]) for k in ("dx", "dw_pre")) and got["df"] is None and got["dgate"] is None
    alone = op.backward(None, c.dn, c.x, **kw)
    assert torch.equal(alone["dx"], op.backward(torch.zeros_like(c.dy), c.dn, c.x, **kw)["dx"])
    del want
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_zeros_and_of_one_value(dt, kind):
    T, D = 6, 130
    op = ResidualNorm(T, D, TYPES[dt], kind=kind, eps=EPS)
    c = Case(T, D, dt, kind)
    c.f[0], c.f[1], c.x[0], c.x[2] = 0, 3, 0, -2
    if kind == "rms":
        c.check(op)
    else:  # a row of one value has no deviation but its mean's rounding
        y, n = op.forward(c.x, c.f, **c.kw)
        assert bool(y.isfinite().all()) and bool(n.isfinite().all())
        assert all(v is None or bool(v.isfinite().all()) for v in op.backward(c.dy, c.dn, y, c.f, **c.kw).values())
        flat, _ = op.forward(torch.zeros_like(c.x), torch.full_like(c.f, 3), pre=False)
        assert float(flat.abs().max()) <= 2.0 ** -21 * 3 / EPS ** 0.5
    op.close()


def test_a_bad_row_stays_alone():
    T, D = 90, 1000
    for dt in TYPES.values():
        op = ResidualNorm(T, D, dt, kind="layer", eps=EPS)
        c = Case(T, D, {v: k for k, v in TYPES.items()}[dt], "layer", group=1)
        y, n, got = c.check(op)
        c.f[11, 4], c.x[50, 0] = float("nan"), float("inf")
        y2, n2 = op.forward(c.x, c.f, **c.kw)
        keep = torch.ones(T, dtype=torch.bool, device="cuda")
        keep[11] = keep[50] = False
        assert torch.equal(y[keep], y2[keep]) and torch.equal(n[keep], n2[keep]) and bool(n2[11].isnan().all()) and not bool(n2[50].isfinite().all())
        got2 = op.backward(c.dy, c.dn, y2, c.f, **c.kw)
        for k in ("dx", "df", "dgate"):
            assert torch.equal(got[k][keep], got2[k][keep]) and bool(got2[k][11].isnan().all())
        op.close()


def test_results_repeat_and_outputs_may_be_inputs():
    T, D = 3000, 1032
    for kind in ("rms", "layer"):
        op = ResidualNorm(T, D, torch.bfloat16, kind=kind, eps=EPS)
        c = Case(T, D, "bf16", kind, group=700)
        y, n, got = c.check(op)
        for _ in range(5):
            y2, n2 = op.forward(c.x, c.f, **c.kw)
            again = op.backward(c.dy, c.dn, y2, c.f, **c.kw)
            assert torch.equal(y, y2) and torch.equal(n, n2) and all(v is None or torch.equal(v, again[k]) for k, v in got.items())
        x = c.x.clone()
        assert op.forward(x, c.f, y=x, **c.kw)[0] is x and torch.equal(x, y)
        dy, f = c.dy.clone(), c.f.clone()
        again = op.backward(dy, c.dn, y, f, out={"dx": dy, "df": f}, **c.kw)
        assert again["dx"] is dy and all(v is None or torch.equal(v, again[k]) for k, v in got.items())
        op.close()


def test_captured_and_replayed():
    T, D = 200, 768
    stream = torch.cuda.Stream()
    op = ResidualNorm(T, D, torch.float32, kind="layer", eps=EPS, stream=stream)
    c = Case(T, D, "f32", "layer", group=30)

    def step():
        y, n = op.forward(c.x, c.f, **c.kw)
        return [y, n] + [v for v in op.backward(c.dy, c.dn, y, c.f, **c.kw).values() if v is not None]

    with torch.cuda.stream(stream):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
    for i in range(2):
        c.x.normal_()
        c.f.normal_()
        torch.cuda.synchronize()
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    del graph
    op.close()


def test_differences():
    """float32 gradients against central differences along random directions: steps of 2^-7 leave a cubic term below 1e-3 of the slope's
    bound, and the loss' rounding (2^-22 of its terms' sizes) below that."""
    T, D = 30, 100
    for kind in ("rms", "layer"):
        op, c = ResidualNorm(T, D, torch.float32, kind=kind, eps=EPS), Case(T, D, "f32", kind, group=4)

        def loss(x, f, **kw):
            y, n = op.forward(x, f, **{**c.kw, **kw})
            return float((y.double() * c.dy.double()).sum() + (n.double() * c.dn.double()).sum())

        y, _ = op.forward(c.x, c.f, **c.kw)
        got = op.backward(c.dy, c.dn, y, c.f, **c.kw)
        for k, g in got.items():
            if g is None:
                continue
            d = torch.randn_like(g)
            d /= d.norm()
            h, ends = 2.0 ** -7, []
            for s in (h, -h):
                x, f, kw = c.x, c.f, {}
                if k == "dx":
                    x = x + s * d
                elif k == "df":
                    f = f + s * d
                else:
                    kw = {k[1:]: c.kw[k[1:]] + s * d}
                ends.append(loss(x, f, **kw))
            assert abs((ends[0] - ends[1]) / (2 * h) - float((g.double() * d.double()).sum())) <= 3e-3 * float(g.double().norm()), (kind, k)
        op.close()


def test_no_rows_and_refusals():
    op = ResidualNorm(8, 40, torch.float32, kind="layer")
    c = Case(4, 40, "f32", "layer")
    y, n = op.forward(c.x[:0], c.f[:0], **c.kw)
    got = op.backward(c.dy[:0], c.dn[:0], y, c.f[:0], out={"dw_post": torch.full((40,), 5.0, device="cuda")}, **c.kw)
    assert y.shape == n.shape == (0, 40) and bool((got["dw_post"] == 0).all()) and bool((got["db_pre"] == 0).all())
    with pytest.raises(ScarError) as e:
        op.forward(torch.zeros(9, 40, device="cuda"))
    assert e.value.code == -7
    rms = ResidualNorm(8, 40, torch.float32, forward_only=True)
    with pytest.raises(ScarError) as e:
        rms.forward(c.x, w_pre=c.kw["w_pre"], b_pre=c.kw["b_pre"])
    assert e.value.code == -1
    with pytest.raises(ScarError) as e:
        rms.backward(c.dy, c.dn, c.x)
    assert e.value.code == -5
    with pytest.raises(ScarError) as e:
        ResidualNorm(8, 16385, torch.float32)
    assert e.value.code == -7
    op.close()
    rms.close()


def test_far_rows():
    """Rows whose offsets pass 2^32 bytes and elements."""
    T, D, far = 3, 264, (1 << 31) + 64
    op = ResidualNorm(T, D, torch.bfloat16)
    c = Case(T, D, "bf16")
    y, n, got = c.check(op)
    buf = torch.empty(2 * far + D, dtype=torch.bfloat16, device="cuda")
    wide = buf.as_strided((T, D), (far, 1))
    wide.copy_(c.x)
    assert all(torch.equal(p, q) for p, q in zip(op.forward(wide, c.f, **c.kw), (y, n)))
    wide.copy_(y)
    out = op.backward(c.dy, c.dn, wide, c.f, **c.kw)
    assert torch.equal(out["df"], got["df"])
    op.backward(c.dy, c.dn, y, c.f, out={"dx": wide}, **c.kw)
    assert torch.equal(wide, got["dx"])
    op.close()


def test_reports_of_a_wait_that_gave_up():
    from paper_1810_07354_b200 import api

    op = ResidualNorm(4, 40, torch.float32)
    x = torch.randn(4, 40, device="cuda")
    op.forward(x)
    op.status()
    api.scar_resnorm_selftest_arm_timeout(op.op)
    op.forward(x)
    with pytest.raises(ScarError) as e:
        op.status()
    assert e.value.code == -6
    op.status()
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("off,more", [(0, 1), (1, 2), (3, 8), (8, 8)])
@pytest.mark.parametrize("T,D", [(5, 40), (33, 1001), (3, 8200)])
def test_results_between_other_values(dt, kind, off, more, T, D):
    """Outputs in the middle of wider rows, wherever these begin: what lies beside them stays, and the results are the same but for the
    order of a row's sum."""
    op = ResidualNorm(T, D, TYPES[dt], kind=kind, eps=EPS)
    c = Case(T, D, dt, kind, group=2)
    y, n = op.forward(c.x, c.f, **c.kw)
    got = op.backward(c.dy, c.dn, y, c.f, **c.kw)
    wide = {k: torch.full((v.shape[0], off + D + more), 7.0, device="cuda", dtype=v.dtype) for k, v in (("y", y), ("n", n), ("dx", y), ("df", y), ("dgate", c.gate))}
    part = {k: v[:, off: off + D] for k, v in wide.items()}
    op.forward(c.x, c.f, y=part["y"], n=part["n"], **c.kw)
    op.backward(c.dy, c.dn, y, c.f, out={k: part[k] for k in ("dx", "df", "dgate")}, **c.kw)
    for k, whole in (("y", y), ("n", n), *((k, got[k]) for k in ("dx", "df", "dgate"))):
        assert float((part[k].double() - whole.double()).norm()) <= 2 * max(unit(TYPES[dt]), 2.0 ** -20) * float(whole.double().norm()), k
        assert bool((wide[k][:, :off] == 7).all()) and bool((wide[k][:, off + D:] == 7).all()), k
    op.close()


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("off,more,group", [(0, 1, 0), (1, 0, 1), (1, 2, 2), (3, 9, 7), (5, 3, 500)])
@pytest.mark.parametrize("T,D", [(1, 9), (2, 1), (40, 3), (37, 70), (700, 513), (350, 1001), (9, 4099), (7, 8195)])
def test_what_lies_beside_the_rows_is_not_used(dt, kind, off, more, group, T, D):
    """Matrices in the middle of wider rows of NaN and infinities, each beginning elsewhere: the bits are those of rows that lie alone."""
    op = ResidualNorm(T, D, TYPES[dt], kind=kind, eps=EPS)
    c = Case(T, D, dt, kind, group=group)

    def beside(v, at):
        if v is None:
            return None
        w = torch.full((v.shape[0], at + D + more + 1), float("nan"), device="cuda", dtype=v.dtype)
        w[:, ::2] = float("inf")
        w[:, at: at + D] = v
        return w[:, at: at + D]

    def odd(v, at):  # the same distance from words, with ordinary values beside them
        return None if v is None else torch.ones(v.shape[0], at + D + more + 1, device="cuda", dtype=v.dtype)[:, at: at + D].copy_(v)

    got = []
    for place in (odd, beside):
        kw = dict(c.kw, gate=place(c.gate, off + 2))
        y, n = op.forward(place(c.x, off), place(c.f, off + 1), **kw)
        g = op.backward(place(c.dy, off), place(c.dn, off + 1), place(y, off), place(c.f, off + 3), **kw)
        got.append([y, n] + [g[k] for k in sorted(g) if g[k] is not None])
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    op.close()
