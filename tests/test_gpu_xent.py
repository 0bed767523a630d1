"""Linear softmax cross entropy and its gradient against the definition in 64 bits.

Tolerances, derived from the formats and the lengths of the sums (nothing here was fitted):

* a product sum over K terms in float32 whose partial sums join at most K/16 + 16 times, each join off by at most one
  unit in the last place: ``gamma(K) = (K/16 + 16) * 2^-23`` of the sum of absolute products;
* a logit is therefore off by ``ez = gamma(D) * max_v sum_d |h||w|``, a probability by the factor ``2 ez`` plus a few
  units of exp, log and the running sum (``2^-20``), and, in the 16-bit types, by the 11 bits it is held in (``2^-11``);
* the gradient of a logit is rounded once to the operands' type (unit ``u``: 2^-8, 2^-11, 2^-23 for the three planes
  of float32); values below ``2^-36`` may vanish;
* a gradient adds ``gamma`` of its own sum and one rounding of the result (float16 also has a smallest step, 2^-25).
"""

import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import LinearCrossEntropy, ScarError, _build, api  # noqa: E402

gpu = pytest.mark.gpu
IGN = -100
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def gamma(k):
    return (k / 16 + 16) * 2.0 ** -23


def make(T, V, D, dtype, seed=0, spread=1.5, ignored=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(V, D, generator=g, device="cuda") * (spread / D ** 0.5)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    h = torch.randn(T, D, generator=g, device="cuda") + (0.5 * w[y] if T else 0.0)
    if ignored:
        y[torch.rand(T, generator=g, device="cuda") < ignored] = IGN
    return h.to(dtype), w.to(dtype), y


def reference(h, w, y, reduction="mean", scale=1.0):
    """The definition in 64 bits with the bounds above for every output."""
    dt = h.dtype
    u = UNIT[dt]
    V, D = w.shape
    kept = (y >= 0) & (y < V)
    h = torch.where(kept[:, None], h, torch.zeros((), dtype=dt, device=h.device)).double()
    w = w.double()
    yc = torch.where(kept, y, torch.zeros_like(y))
    z = h @ w.T
    lse = torch.logsumexp(z, 1)
    zl = z.gather(1, yc[:, None])[:, 0]
    row = torch.where(kept, lse - zl, torch.zeros_like(lse))
    n = max(1, int(kept.sum())) if reduction == "mean" else 1
    loss = row.sum() / n
    p = torch.exp(z - lse[:, None]) * kept[:, None]
    dz = p.clone()
    if len(y):
        dz.scatter_add_(1, yc[:, None], torch.where(kept, -1.0, 0.0).double()[:, None])
    g = scale / n
    ez = gamma(D) * (h.abs() @ w.abs().T).amax(1) if len(y) else lse
    e_row = 2 * ez + 2.0 ** -20 * (1 + lse.abs() + zl.abs())
    held = 0.0 if dt == torch.float32 else 2.0 ** -11
    e_dz = p * (2 * ez[:, None] + held + 2.0 ** -20) + u * dz.abs() + 2.0 ** -36 * kept[:, None]
    dh, dw = dz @ w * g, dz.T @ h * g
    tiny = 2.0 ** -24 if dt == torch.float16 else 0.0
    e_dh = abs(g) * (e_dz @ w.abs() + gamma(V) * (dz.abs() @ w.abs())) + u * dh.abs() + tiny
    e_dw = abs(g) * (e_dz.T @ h.abs() + gamma(len(y)) * (dz.abs().T @ h.abs())) + u * dw.abs() + tiny
    e_loss = (torch.where(kept, e_row, torch.zeros_like(e_row)).sum() / n) + 2.0 ** -22 * loss.abs()
    return dict(loss=loss, row=row, dh=dh, dw=dw), dict(loss=e_loss, row=e_row, dh=e_dh, dw=e_dw), int(kept.sum())


def close(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float((off / tol.clamp(min=1e-300)).max()):.3g} of the bound"


def check(op, h, w, y, reduction="mean", scale=1.0, **kw):
    want, tol, n = reference(h, w, y, reduction, scale)
    loss, row = op.loss(h, w, y)
    close(row, want["row"], tol["row"], "row loss without gradients")
    close(loss, want["loss"], tol["loss"], "loss without gradients")
    loss, row, dh, dw = op.loss_and_grad(h, w, y, grad_scale=scale, **kw)
    info = op.status()
    assert int(info.rows) == n and info.loss == float(loss)
    close(row, want["row"], tol["row"], "row loss")
    close(loss, want["loss"], tol["loss"], "loss")
    close(dh, want["dh"], tol["dh"], "dh")
    close(dw, want["dw"], tol["dw"], "dw")
    if n >= 16 and scale == 1.0:  # as a whole: two roundings, each 0.43 units in the mean square
        u = max(UNIT[h.dtype], 2.0 ** -18)
        tiny = 2.0 ** -25 if h.dtype == torch.float16 else 0.0
        for a, b in ((dh, want["dh"]), (dw, want["dw"])):
            if float(b.abs().max()) < 2.0 ** -36:
                continue  # all of it may vanish (the bound of each value above says so)
            assert float((a.double() - b).norm()) <= u * float(b.norm()) + tiny * b.numel() ** 0.5
    return loss, row, dh, dw


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,V,D", [
    (1, 1, 1), (1, 2, 3), (2, 1, 8), (3, 5, 7), (1, 1000, 64), (16, 256, 64), (63, 255, 65), (64, 257, 128), (65, 300, 100),
    (127, 513, 72), (128, 1000, 1000), (129, 4099, 200), (257, 33, 520), (300, 777, 129), (511, 1030, 264), (1030, 100, 40),
    (5, 40000, 48), (700, 3, 16), (17, 130, 5000), (256, 10, 9001),
])
def test_every_output_is_within_its_bound(dt, T, V, D):
    h, w, y = make(T, V, D, TYPES[dt], seed=T + V + D, ignored=0.2 if T > 20 else 0.0)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    check(op, h, w, y)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_larger_sizes(dt):
    T, V, D = 1200, 20011, 1024
    h, w, y = make(T, V, D, TYPES[dt], seed=3, ignored=0.1)
    op = LinearCrossEntropy(T + 500, V, D, TYPES[dt])
    check(op, h, w, y)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,V,D,ignored", [
    (2500, 300, 64, 0.1), (5000, 9000, 40, 0.3), (4800, 120, 1000, 0.0),  # a warp per row of the softmax; rows listed by a kernel of their own
    (3000, 1500, 72, 0.95),  # far fewer rows count than the launch was made for
    (12, 30000, 96, 0.0),    # few long rows: cut into ranges
    (40, 260, 6000, 0.2),    # few tiles: the sum over D is cut into parts
    (700, 60000, 24, 0.1),   # dh sums over very many classes
    (9000, 40, 48, 0.2),     # dw sums over very many rows
])
def test_every_way_through_the_kernels(dt, T, V, D, ignored):
    h, w, y = make(T, V, D, TYPES[dt], seed=T + D, ignored=ignored)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    check(op, h, w, y)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,V,D", [(300, 260, 6000), (700, 60_000, 24), (6000, 40, 48), (1100, 520, 2000)])
def test_parts_of_split_sums_for_any_number_of_rows_that_count(dt, T, V, D):
    """Products whose sums are cut into parts, launched for T rows while from none to all of them count: the kernel that
    joins the parts takes as many as there are."""
    h, w, y = make(T, V, D, TYPES[dt], seed=V)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    for kept in sorted({0, 1, 2, 63, 64, 65, 255, 256, 257, T // 4, T // 2, T - 1, T}):
        some = y.clone()
        g = torch.Generator(device="cuda").manual_seed(kept)
        some[torch.randperm(T, generator=g, device="cuda")[kept:]] = IGN
        check(op, h, w, some)
    op.close()


@gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_offsets_beyond_32_bits(dt):
    """w and dw of 2.4e9 values: rows behind the 2^31st and the 2^32nd value's byte are checked against the definition."""
    T, V, D = 6, 300_000, 8000
    w = torch.empty(V, D, dtype=TYPES[dt], device="cuda").normal_(std=1.5 / D ** 0.5)
    g = torch.Generator(device="cuda").manual_seed(1)
    y = torch.tensor([0, V - 1, 268_435, 268_436, IGN, V - 2], device="cuda")
    h = torch.randn(T, D, generator=g, device="cuda").to(TYPES[dt])
    op = LinearCrossEntropy(T, V, D, TYPES[dt], reduction="sum")
    loss, row, dh, dw = op.loss_and_grad(h, w, y)
    kept = y >= 0
    hd = torch.where(kept[:, None], h, torch.zeros_like(h)).double()
    z = torch.cat([hd @ c.double().T for c in w.split(20_000)], 1)
    lse = torch.logsumexp(z, 1)
    want = torch.where(kept, lse - z.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    ez = 2 * gamma(D) * 50 + 2.0 ** -18
    assert bool(((row.double() - want).abs() <= ez).all())
    p = torch.exp(z - lse[:, None]) * kept[:, None]
    p[torch.arange(T), y.clamp(min=0)] -= kept.double()
    rows = torch.cat([torch.arange(0, 3), torch.arange(268_430, 268_440), torch.arange(V - 3, V)]).cuda()
    u = UNIT[TYPES[dt]]
    ref = p.T[rows] @ hd
    tol = (u + 2.0 ** -11 + 2 * ez) * (p.T[rows].abs() @ hd.abs()) + u * ref.abs() + 2.0 ** -24
    assert bool(((dw[rows].double() - ref).abs() <= tol).all())
    ref = sum(p[:, i: i + 20_000] @ w[i: i + 20_000].double() for i in range(0, V, 20_000))
    assert float((dh.double() - ref).norm()) <= u * float(ref.norm()) and not dh[4].any()
    op.close()


@gpu
def test_float32_offsets_beyond_32_bits():
    """2.4e9 float32 values of w and dw, three planes of which are 14.4 GB: rows behind the 2^31st value and behind the
    2^32nd byte, of w, of a plane and of dw, against the definition."""
    T, V, D = 6, 300_000, 8000
    w = torch.empty(V, D, device="cuda").normal_(std=1.5 / D ** 0.5)
    g = torch.Generator(device="cuda").manual_seed(1)
    y = torch.tensor([0, V - 1, 268_435, 134_217, IGN, V - 2], device="cuda")
    h = torch.randn(T, D, generator=g, device="cuda")
    op = LinearCrossEntropy(T, V, D, torch.float32, reduction="sum")
    loss, row, dh, dw = op.loss_and_grad(h, w, y)
    assert torch.equal(op.loss(h, w, y)[1], row)
    kept = y >= 0
    hd = torch.where(kept[:, None], h, torch.zeros_like(h)).double()
    z = torch.cat([hd @ c.double().T for c in w.split(20_000)], 1)
    lse = torch.logsumexp(z, 1)
    want = torch.where(kept, lse - z.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    ez = 2 * gamma(D) * 50 + 2.0 ** -18
    assert bool(((row.double() - want).abs() <= ez).all())
    p = torch.exp(z - lse[:, None]) * kept[:, None]
    p[torch.arange(T), y.clamp(min=0)] -= kept.double()
    rows = torch.cat([torch.arange(0, 3), torch.arange(134_210, 134_225), torch.arange(268_430, 268_440), torch.arange(V - 3, V)]).cuda()
    u = UNIT[torch.float32]
    ref = p.T[rows] @ hd
    tol = (u + 2 * ez) * (p.T[rows].abs() @ hd.abs()) + u * ref.abs() + 2.0 ** -36
    assert bool(((dw[rows].double() - ref).abs() <= tol).all())
    ref = sum(p[:, i: i + 20_000] @ w[i: i + 20_000].double() for i in range(0, V, 20_000))
    assert float((dh.double() - ref).norm()) <= 2.0 ** -18 * float(ref.norm()) and not dh[4].any()
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_counts_of_rows_that_do_not_count(dt):
    T, V, D = 40, 200, 72
    h, w, good = make(T, V, D, TYPES[dt])
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    for y, want in ((torch.full((T,), IGN, device="cuda"), (0, T, 0)), (torch.full((T,), V, device="cuda"), (0, 0, T)), (torch.full((T,), -1, device="cuda"), (0, 0, T)),
                    (torch.full((T,), 2 ** 40, device="cuda"), (0, 0, T)), (torch.cat([good[:30], torch.tensor([IGN] * 7 + [-1, V, -2 ** 62], device="cuda")]), (30, 7, 3))):
        for call in (op.loss, op.loss_and_grad):
            call(h, w, y)
            info = op.status()
            assert (int(info.rows), int(info.ignored), int(info.bad)) == want
    op.close()
    T = 3000  # listed by a kernel of their own
    h, w, y = make(T, V, D, TYPES[dt])
    y[::3], y[1::300] = IGN, V
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    op.loss(h, w, y)
    info = op.status()
    assert (int(info.rows), int(info.ignored), int(info.bad)) == (1990, 1000, 10)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_sum_and_scale(dt):
    h, w, y = make(70, 600, 96, TYPES[dt], seed=5, ignored=0.3)
    op = LinearCrossEntropy(70, 600, 96, TYPES[dt], reduction="sum")
    check(op, h, w, y, reduction="sum")
    check(op, h, w, y, reduction="sum", scale=-0.37)
    check(op, h, w, y, reduction="sum", scale=0.0)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,V,D", [(1000, 500, 64), (1300, 4100, 136), (600, 70, 2000), (900, 301, 67), (520, 2000, 1001)])
def test_pieces_of_rows_give_what_all_rows_at_once_give(dt, T, V, D):
    """A small workspace forces several pieces (256 rows each), the last one short; ignored rows shift the others."""
    h, w, y = make(T, V, D, TYPES[dt], seed=9, ignored=0.25)
    y[:300] = IGN  # a piece's worth: the last piece of the call has no row left
    op = LinearCrossEntropy(T, V, D, TYPES[dt], workspace_bytes=1)
    check(op, h, w, y)
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("D", [64, 67])
def test_strided_and_unaligned_operands_and_untouched_gaps(dt, D):
    T, V, dtype = 90, 333, TYPES[dt]
    h0, w0, y = make(T, V, D, dtype, seed=2, ignored=0.1)
    op = LinearCrossEntropy(T, V, D, dtype)
    want = check(op, h0, w0, y)
    for lead, gap in ((0, 0), (1, 0), (0, 5), (3, 9), (8, 64 - D % 64)):
        def place(m):
            buf = torch.full((lead + m.shape[0] * (D + gap) + 7,), 7.0, dtype=dtype, device="cuda")
            v = buf[lead: lead + m.shape[0] * (D + gap)].view(m.shape[0], D + gap)[:, :D]
            v.copy_(m)
            return buf, v
        (_, h), (_, w) = place(h0), place(w0)
        (bh, dh), (bw, dw) = place(torch.zeros_like(h0)), place(torch.zeros_like(w0))
        got = op.loss_and_grad(h, w, y, dh=dh, dw=dw)
        for a, b in zip(got, want):
            assert torch.equal(a, b), "where the operands lie changes nothing"
        for buf, v in ((bh, dh), (bw, dw)):
            left = buf.clone()
            left[lead: lead + v.shape[0] * (D + gap)].view(v.shape[0], D + gap)[:, :D] = 7.0
            assert bool((left == 7.0).all()), "bytes between and around the rows were written"
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("D", [64, 72, 67])
def test_every_operand_off_its_boundary_by_itself(dt, D):
    """h, w, dh and dw each moved by one element while the others lie on 16-byte boundaries: the same bits."""
    T, V, dtype = 130, 600, TYPES[dt]
    h, w, y = make(T, V, D, dtype, seed=13, ignored=0.2)
    op = LinearCrossEntropy(T, V, D, dtype)
    want = check(op, h, w, y)

    def moved(m):
        buf = torch.full((m.numel() + 9,), 7.0, dtype=dtype, device="cuda")
        v = buf[1: 1 + m.numel()].view_as(m)
        v.copy_(m)
        return buf, v

    for which in range(4):
        ops = [h, w, torch.empty_like(h), torch.empty_like(w)]
        buf, ops[which] = moved(ops[which])
        got = op.loss_and_grad(ops[0], ops[1], y, dh=ops[2], dw=ops[3])
        for a, b in zip(got, want):
            assert torch.equal(a, b), which
        assert float(buf[0]) == 7.0 and bool((buf[-8:] == 7.0).all())
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_no_row_counts(dt):
    T, V, D = 40, 200, 72
    h, w, _ = make(T, V, D, TYPES[dt])
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    for y in (torch.full((T,), IGN, device="cuda"), torch.full((T,), V, device="cuda"), torch.full((T,), -1, device="cuda")):
        loss, row, dh, dw = op.loss_and_grad(h, w, y)
        info = op.status()
        assert (int(info.rows), int(info.ignored), int(info.bad)) == (0, T, 0) if int(y[0]) == IGN else (0, 0, T)
        assert float(loss) == 0.0 and not row.any() and not dh.any() and not dw.any()
        loss, row = op.loss(h, w, y)
        assert float(loss) == 0.0 and not row.any()
    empty = op.loss_and_grad(h[:0], w, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert float(empty[0]) == 0.0 and empty[1].numel() == 0 and not empty[3].any()
    assert float(op.loss(h[:0], w, torch.empty(0, dtype=torch.int64, device="cuda"))[0]) == 0.0
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_what_ignored_rows_hold_reaches_nothing(dt):
    T, V, D = 150, 700, 128
    h, w, y = make(T, V, D, TYPES[dt], seed=8, ignored=0.4)
    y[0], y[-1] = IGN, V + 5
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    want = check(op, h, w, y)
    out = (y < 0) | (y >= V)
    for v in (float("nan"), float("inf"), float("-inf"), float(torch.finfo(TYPES[dt]).min)):
        g = h.clone()
        g[out] = v
        for a, b in zip(op.loss_and_grad(g, w, y), want):
            assert torch.equal(a, b)
    assert int(op.status().bad) == 1 and int(op.status().rows) == int((~out).sum())
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_nonfinite_rows_stay_in_their_rows(dt):
    """A NaN or an infinity in a row that counts spoils that row's loss (as the formula says) and no other row's."""
    T, V, D = 140, 600, 64
    h, w, y = make(T, V, D, TYPES[dt], seed=4)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    _, row0, dh0, _ = op.loss_and_grad(h, w, y)
    g = h.clone()
    g[3, 5], g[77, 0], g[130, 63] = float("nan"), float("inf"), float("-inf")
    loss, row, dh, dw = op.loss_and_grad(g, w, y)
    hit = torch.zeros(T, dtype=torch.bool, device="cuda")
    hit[[3, 77, 130]] = True
    assert bool(row[hit].isnan().all()) and torch.equal(row[~hit], row0[~hit]) and bool(loss.isnan())
    assert bool(dh[hit].isnan().any(1).all()) and torch.equal(dh[~hit], dh0[~hit])
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_logits_far_apart(dt):
    """Large logits: probabilities of exactly one and zero, and a whole group of classes at minus infinity."""
    T, V, D = 64, 1500, 32
    h, w, y = make(T, V, D, TYPES[dt], seed=6, spread=60.0)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    check(op, h, w, y)  # every label's probability is one: the gradients vanish
    check(op, h, w, (y + 1) % V)  # every label's probability is next to zero: they are as large as they get
    if dt != "f16":  # (-1e38) * 60 overflows float32 to -inf in the logit itself
        h = torch.zeros(T, D, dtype=TYPES[dt], device="cuda")
        h[:, 0] = 60.0
        w = torch.zeros(V, D, dtype=TYPES[dt], device="cuda")
        w[200:900, 0] = -1e38
        y = torch.randint(0, 200, (T,), device="cuda")
        loss, row, dh, dw = op.loss_and_grad(h, w, y)
        want = float(np.log(V - 700))
        assert bool(((row - want).abs() <= 1e-5 * want).all())
        assert not dw[200:900].any() and bool(dw.isfinite().all())
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_equal_inputs_give_equal_bits(dt):
    h, w, y = make(333, 2222, 192, TYPES[dt], seed=1, ignored=0.1)
    op = LinearCrossEntropy(333, 2222, 192, TYPES[dt])
    first = op.loss_and_grad(h, w, y)
    for _ in range(20):
        for a, b in zip(op.loss_and_grad(h, w, y), first):
            assert torch.equal(a, b)
    op.close()


@gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,V,D", [
    (48, 60_000, 72), (20, 90_000, 24), (64, 40_000, 264), (30, 30_000, 520),  # dw: the last columns fill half a stage, on every tile
    (1500, 30_017, 64), (700, 20_001, 128), (300, 45_031, 96),                 # exponentials: the same, and row tiles that end early
])
def test_results_stored_while_the_next_ones_are_staged(dt, T, V, D):
    """Many tiles per CTA pair whose products take less time than their results: each of them waits for the stage that the
    one before is still stored from.  Every value within its bound, and the same bits every time."""
    h, w, y = make(T, V, D, TYPES[dt], seed=T + D)
    op = LinearCrossEntropy(T, V, D, TYPES[dt])
    first = check(op, h, w, y)
    dh, dw, row = torch.empty_like(h), torch.empty_like(w), torch.empty(T, device="cuda")
    for _ in range(30):
        dw.fill_(7.0)
        op.loss_and_grad(h, w, y, row_loss=row, dh=dh, dw=dw)
        assert torch.equal(row, first[1]) and torch.equal(dh, first[2]) and torch.equal(dw, first[3])
    op.close()


@gpu
def test_gradient_against_differences():
    """Central differences of the float32 operator's own loss along random directions.  The loss is smooth with a third
    derivative of order one along a unit step; with a step of 2^-5 the truncation is below 2^-10 / 6 and the rounding
    below 2^-20 * |loss| / 2^-5."""
    T, V, D = 60, 301, 50
    h, w, y = make(T, V, D, torch.float32, seed=11, ignored=0.1)
    op = LinearCrossEntropy(T, V, D, torch.float32)
    _, _, dh, dw = op.loss_and_grad(h, w, y)
    g = torch.Generator(device="cuda").manual_seed(12)
    step = 2.0 ** -5
    for _ in range(6):
        a = torch.randn(T, D, generator=g, device="cuda")
        b = torch.randn(V, D, generator=g, device="cuda")
        a, b = a / a.norm(), b / b.norm()
        up, down = float(op.loss(h + step * a, w + step * b, y)[0]), float(op.loss(h - step * a, w - step * b, y)[0])
        slope = float((dh.double() * a).sum() + (dw.double() * b).sum())
        assert abs((up - down) / (2 * step) - slope) <= 2.0 ** -10 / 6 + 2.0 ** -15 * 8
    op.close()


@gpu
def test_another_stream_and_a_captured_graph():
    T, V, D = 200, 1000, 128
    h, w, y = make(T, V, D, torch.bfloat16, seed=7)
    op = LinearCrossEntropy(T, V, D, torch.bfloat16)
    want = op.loss_and_grad(h, w, y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        h2 = h * 1
        got = op.loss_and_grad(h2, w, y)
        total = [x.double().sum() for x in got]
    side.synchronize()
    for a, b, t in zip(got, want, total):
        assert torch.equal(a, b) and float(t) == float(b.double().sum())
    with torch.cuda.stream(side):
        mine = LinearCrossEntropy(T, V, D, torch.bfloat16)
        dh, dw, row = torch.empty_like(h), torch.empty_like(w), torch.empty(T, device="cuda")
        mine.loss_and_grad(h, w, y, row_loss=row, dh=dh, dw=dw)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mine.loss_and_grad(h, w, y, row_loss=row, dh=dh, dw=dw)
        for x in (dh, dw, row):
            x.zero_()
        graph.replay()
    side.synchronize()
    assert torch.equal(dh, want[2]) and torch.equal(dw, want[3]) and torch.equal(row, want[1])
    op.close()
    mine.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,V,D,room", [(200, 1000, 128, 0), (700, 500, 64, 1), (40, 260, 6000, 0), (3000, 300, 64, 0)])
def test_a_wait_that_gave_up_shows_in_the_loss(dt, T, V, D, room):
    """A caller that reads no status sees a NaN; the call after it is a whole one.  (No wait is made to run out: the hook
    sets the flag that one would set.)"""
    h, w, y = make(T, V, D, TYPES[dt], seed=4, ignored=0.1)
    op = LinearCrossEntropy(T, V, D, TYPES[dt], workspace_bytes=room)
    want = op.loss_and_grad(h, w, y)
    alone = op.loss(h, w, y)
    for call in (op.loss_and_grad, op.loss):
        api.scar_xent_selftest_arm_timeout(op.op)
        assert bool(call(h, w, y)[0].isnan())
        with pytest.raises(ScarError) as e:
            op.status()
        assert e.value.code == -6
    assert all(torch.equal(a, b) for a, b in zip(op.loss_and_grad(h, w, y), want))
    assert all(torch.equal(a, b) for a, b in zip(op.loss(h, w, y), alone)) and op.status().loss == float(alone[0])
    op.close()


@gpu
def test_refusals_leave_everything_untouched():
    T, V, D = 8, 40, 16
    h, w, y = make(T, V, D, torch.bfloat16)
    op = LinearCrossEntropy(T, V, D, torch.bfloat16)
    with pytest.raises(ScarError):
        op.status()  # nothing ran yet
    with pytest.raises(ScarError):
        op.loss(torch.cat([h, h]), w, torch.cat([y, y]))  # more rows than the handle was made for
    with pytest.raises(TypeError):
        op.loss(h.float(), w, y)
    with pytest.raises(TypeError):
        op.loss(h, w, y.int())
    with pytest.raises(ValueError):
        op.loss(h, w[:-1], y)
    with pytest.raises(ValueError):
        op.loss(h.T.contiguous().T, w, y)
    with pytest.raises(ScarError):
        op.loss(h[:1].expand(T, D), w, y)  # rows on top of each other
    with pytest.raises(TypeError):
        LinearCrossEntropy(T, V, D, torch.float64)
    lib, a = api.load_library(), h.data_ptr()
    fixed = torch.full((V, D), 3.0, dtype=torch.bfloat16, device="cuda")
    bad = [(a + 1, D, w.data_ptr(), D, y.data_ptr(), T), (a, D - 1, w.data_ptr(), D, y.data_ptr(), T), (None, D, w.data_ptr(), D, y.data_ptr(), T),
           (a, D, None, D, y.data_ptr(), T), (a, D, w.data_ptr(), D, None, T), (a, D, w.data_ptr(), D, y.data_ptr() + 4, T)]
    for args in bad:
        assert lib.scar_xent_loss(op.op, *args, None, None) == -1
        assert lib.scar_xent_loss_grad(op.op, *args, 1.0, None, None, fixed.data_ptr(), D, fixed.data_ptr(), D) == -1
    good = (a, D, w.data_ptr(), D, y.data_ptr(), T)
    assert lib.scar_xent_loss_grad(op.op, *good, 1.0, None, None, None, D, fixed.data_ptr(), D) == -1
    assert lib.scar_xent_loss_grad(op.op, *good, 1.0, None, None, fixed.data_ptr(), D, None, D) == -1
    assert lib.scar_xent_loss_grad(op.op, *good, 1.0, None, None, fixed.data_ptr(), D, fixed.data_ptr(), D - 1) == -1
    small = LinearCrossEntropy(T, V, D, torch.bfloat16, loss_only=True)
    assert lib.scar_xent_loss_grad(small.op, *good, 1.0, None, None, fixed.data_ptr(), D, fixed.data_ptr(), D) == -5
    assert small.workspace_bytes() <= op.workspace_bytes()
    assert float(small.loss(h, w, y)[0]) == float(op.loss(h, w, y)[0])
    torch.cuda.synchronize()
    assert bool((fixed == 3.0).all())
    op.close()
    small.close()


@gpu
def test_host_tensors_are_refused():
    T, V, D = 8, 40, 16
    h, w, y = make(T, V, D, torch.float32)
    op = LinearCrossEntropy(T, V, D, torch.float32)
    with pytest.raises(ValueError):
        op.loss(h, w, y, row_loss=torch.empty(T))
    for args in ((h.cpu(), w, y), (h, w.cpu(), y), (h, w, y.cpu())):
        with pytest.raises(TypeError):
            op.loss(*args)
    with pytest.raises(TypeError):
        op.loss_and_grad(h, w, y, dh=torch.empty(T, D))
    with pytest.raises(TypeError):
        op.loss_and_grad(h, w, y, dw=torch.empty(V, D))
    assert api.scar_xent_launch_count(op.op) == 0
    op.close()


@gpu
def test_results_off_their_boundary_and_rows_too_far_apart_are_refused():
    T, V, D = 8, 40, 16
    h, w, y = make(T, V, D, torch.bfloat16)
    op = LinearCrossEntropy(T, V, D, torch.bfloat16)
    lib, room = api.load_library(), torch.full((64 + V * D,), 3.0, device="cuda")
    a, good = room.data_ptr(), (h.data_ptr(), D, w.data_ptr(), D, y.data_ptr(), T)
    for row, loss in ((a + 2, a + 64), (a + 1, None), (a, a + 65), (None, a + 66)):
        assert lib.scar_xent_loss(op.op, *good, row, loss) == -1
        assert lib.scar_xent_loss_grad(op.op, *good, 1.0, row, loss, a + 256, D, a + 512, D) == -1
    for dhp, dwp in ((1 << 38, D), (D, 1 << 38)):
        assert lib.scar_xent_loss_grad(op.op, *good, 1.0, None, None, a + 256, dhp, a + 512, dwp) == -1
    assert api.scar_xent_launch_count(op.op) == 0
    torch.cuda.synchronize()
    assert bool((room == 3.0).all())
    op.close()


def test_arguments_are_checked_before_any_device_work():
    _build.build()
    lib = api.load_library()
    op = C.c_void_p(5)
    good = dict(max_tokens=8, n_classes=4, dim=4, ignore_label=IGN, workspace_bytes=0, dtype=2, reduction=0, loss_only=0)
    assert lib.scar_xent_init(None, C.byref(api.scar_xent_config(**good)), None) == -1
    assert lib.scar_xent_init(C.byref(op), None, None) == -1 and op.value is None
    for change in (dict(dtype=1), dict(dtype=9), dict(reduction=2), dict(n_classes=0), dict(dim=0), dict(n_classes=1 << 31),
                   dict(dim=1 << 31), dict(max_tokens=1 << 31)):
        assert lib.scar_xent_init(C.byref(op), C.byref(api.scar_xent_config(**{**good, **change})), None) == -1
    assert lib.scar_xent_loss(None, None, 0, None, 0, None, 0, None, None) == -1
    assert lib.scar_xent_loss_grad(None, None, 0, None, 0, None, 0, 1.0, None, None, None, 0, None, 0) == -1
    assert lib.scar_xent_status(None, None) == -1 and lib.scar_xent_destroy(None) == -1
    assert lib.scar_xent_workspace_bytes(None) == 0 and lib.scar_xent_launch_count(None) == 0
    ctx, layout = C.c_void_p(), api.make_layout(1024, 0, 256, 8)
    for dt in (api.SCAR_BF16, api.SCAR_F16):  # operand types of these operators only
        assert lib.scar_ckpt_init(C.byref(ctx), 0x1000, dt, C.byref(layout), None) == -1


def test_the_hook_checks_its_argument():
    _build.build()
    assert api.load_library().scar_xent_selftest_arm_timeout(None) == -1
