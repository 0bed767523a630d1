"""Global gradient norm and clipping against the formulas in 64 bits.

Tolerances: a float32 running sum takes at most 2^14 terms of one piece of 32 KiB spread over hundreds of lanes (at
most 128 terms a lane: 128 * 2^-24 < 2^-17 relative on a sum of squares or magnitudes), everything beyond is double;
the returned float32 adds 2^-24.  The factor is a float32 (2^-24), its product is rounded once to the type."""

import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")

from paper_1810_07354_b200 import GradientNorm, ScarError, _build, api  # noqa: E402

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SUM_TOL = 2.0 ** -17


def tensors(lengths, types, seed=0, lead=(0,), scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(lengths):
        at = lead[i % len(lead)]
        buf = torch.randn(at + n + 16, generator=g, device="cuda").mul_(scale * (1 + i % 5)).to(types[i % len(types)])
        out.append(buf[at: at + n])
    return out


def exact_norm(ts, kind):
    if kind == "l2":
        return math.sqrt(math.fsum(float(t.double().square().sum()) for t in ts))
    if kind == "l1":
        return math.fsum(float(t.double().abs().sum()) for t in ts)
    return max([float(t.double().abs().max()) for t in ts if t.numel()], default=0.0)


def check(ts, kind="l2", fraction=0.4, lead=(0,)):
    want = exact_norm(ts, kind)
    tol = 0.0 if kind == "max" else SUM_TOL
    outs = []
    for i, t in enumerate(ts):
        at = lead[i % len(lead)]
        outs.append(torch.full((at + t.numel() + 16,), 7.0, dtype=t.dtype, device="cuda"))
    views = [o[lead[i % len(lead)]: lead[i % len(lead)] + t.numel()] for i, (o, t) in enumerate(zip(outs, ts))]
    keep = [t.clone() for t in ts]
    op = GradientNorm(ts, out=views, kind=kind)
    got = float(op.norm())
    assert abs(got - want) <= (tol + 2.0 ** -23) * want
    assert all(bool((o == 7.0).all()) for o in outs), "the norm alone writes nothing"
    max_norm = fraction * want
    assert float(op.clip(max_norm)) == got
    info = op.status()
    coef = min(1.0, max_norm / want) if want else 1.0
    assert abs(info.norm - want) <= (tol + 2.0 ** -40) * want and abs(info.coef - coef) <= (tol + 2.0 ** -22) * coef
    for i, (t, k, o, v) in enumerate(zip(ts, keep, outs, views)):
        assert torch.equal(t, k), "the input is only read"
        at = lead[i % len(lead)]
        assert bool((o[:at] == 7.0).all()) and bool((o[at + t.numel():] == 7.0).all()), "written outside an output"
        if t.numel():
            x = t.double() * coef
            u = UNIT[t.dtype]
            tiny = 2.0 ** -24 if t.dtype == torch.float16 else 0.0
            assert bool(((v.double() - x).abs() <= (u + tol + 2.0 ** -21) * x.abs() + tiny).all())
    # in place, with the same bits
    place = [torch.empty(lead[i % len(lead)] + t.numel() + 16, dtype=t.dtype, device="cuda")[lead[i % len(lead)]:][: t.numel()] for i, t in enumerate(ts)]
    for p, t in zip(place, ts):
        p.copy_(t)
    inp = GradientNorm(place, kind=kind)
    assert float(inp.clip(max_norm)) == got
    for p, v in zip(place, views):
        assert torch.equal(p, v)
    op.close()
    inp.close()


LISTS = {
    "one element": [1], "two": [2, 1], "zeros among them": [0, 5, 0, 0, 3, 0], "around a vector": list(range(1, 40)),
    "around a piece": [8191, 8192, 8193, 16383, 16384, 16385], "long": [3_000_001], "long and short": [1_000_003, 1, 7, 500_000, 0, 33],
    "many": [(i * 37) % 1000 + 1 for i in range(1500)],
    "as many pieces as are resident": [4096 * 592], "one more": [4096 * 592, 5], "hundreds of short ones": [100 + i for i in range(590)],
}


@gpu
@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clip(name, dt, kind):
    types = list(TYPES.values()) if dt == "mixed" else [TYPES[dt]]
    lead = (0, 1, 3, 8)
    check(tensors(LISTS[name], types, seed=len(name), lead=lead, scale=1e-2), kind, lead=lead)


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_inputs_and_outputs_at_different_offsets(dt):
    for a, b in ((0, 1), (1, 0), (1, 2), (3, 5), (8, 4)):
        lengths = [1, 15, 16, 17, 1000, 40_001]
        check(tensors(lengths, [TYPES[dt]], seed=a * 10 + b, lead=(a,)), lead=(b,))


@gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_a_tensor_beyond_32_bits(dt):
    """2^31 + 77 values (4 GB): a few of them large, at places a 32-bit offset would miss; the rest zero."""
    n = 2 ** 31 + 77
    t = torch.zeros(n, dtype=TYPES[dt], device="cuda")
    at = [0, 2 ** 30 - 1, 2 ** 31 - 1, 2 ** 31, n - 1]
    for i in at:
        t[i] = 3.0
    op = GradientNorm([t])
    want = math.sqrt(9.0 * len(at))
    assert abs(float(op.clip(want / 3)) - want) <= 1e-6 * want
    assert all(float(t[i]) == 1.0 for i in at) and abs(float(op.norm()) - want / 3) <= 1e-6 * want
    op.close()


@gpu
def test_no_tensors_and_no_elements():
    for ts in ([], [torch.empty(0, device="cuda")], [torch.empty(0, device="cuda", dtype=torch.bfloat16)] * 3):
        op = GradientNorm(ts)
        assert float(op.norm()) == 0.0 and float(op.clip(1.0)) == 0.0
        assert op.status().coef == 1.0 and op.status().nonfinite == 0
        op.close()


@gpu
@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
def test_zero_gradients_and_limits(kind):
    ts = [torch.zeros(1000, device="cuda"), torch.zeros(3, dtype=torch.float16, device="cuda")]
    op = GradientNorm(ts, kind=kind)
    for limit in (0.0, 1.0, math.inf):
        assert float(op.clip(limit)) == 0.0 and op.status().coef == 1.0
        assert all(not t.any() for t in ts)
    op.close()
    t = torch.tensor([3.0, -4.0], device="cuda")
    op = GradientNorm([t], kind=kind)
    norm = {"l2": 5.0, "l1": 7.0, "max": 4.0}[kind]
    assert float(op.clip(math.inf)) == norm and t.tolist() == [3.0, -4.0]
    assert float(op.clip(norm)) == norm and t.tolist() == [3.0, -4.0], "a norm at the limit is left alone"
    assert float(op.clip(0.0)) == norm and t.tolist() == [0.0, -0.0]
    op.close()


@gpu
@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
@pytest.mark.parametrize("dt", list(TYPES))
def test_nonfinite_values(dt, kind):
    ts = tensors([1000, 50_000, 3], [TYPES[dt]], seed=1)
    out = [torch.empty_like(t) for t in ts]
    ts[1][777] = float("nan")
    op = GradientNorm(ts, out=out, kind=kind)
    assert math.isnan(float(op.clip(1.0))) and op.status().nonfinite == 1
    assert all(bool(o.isnan().all()) for o in out)
    ts[1][777] = float("-inf")
    assert float(op.clip(1.0)) == math.inf and op.status().nonfinite == 1 and op.status().coef == 0.0
    bad = torch.zeros(50_000, dtype=torch.bool, device="cuda")
    bad[777] = True
    assert bool(out[1][bad].isnan().all()) and not out[1][~bad].any() and not out[0].any()
    op.close()


@gpu
def test_values_whose_squares_leave_float32():
    """The square of 1e30 is not a float32; the sum of squares is held where it is a number."""
    t = torch.full((5000,), 1e30, device="cuda")
    op = GradientNorm([t], kind="l1")
    assert abs(float(op.norm()) - 5e33) <= 1e-5 * 5e33
    op.close()
    op = GradientNorm([t], kind="max")
    assert float(op.norm()) == float(torch.tensor(1e30))
    op.close()


@gpu
@pytest.mark.parametrize("lengths", [[5000, 3, 17], [3_000_001, 40, 0, 777_777]], ids=["one launch", "two launches"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e30, 3e38, 1e-15, 1e-19, 1e-21, 1e-25, 1e-30, 1e-38])
def test_l2_of_values_whose_squares_leave_float32(size, dt, lengths):
    """The squares of these values are no float32, or have lost their bits; the norm is an ordinary one."""
    g = torch.Generator(device="cuda").manual_seed(2)
    ts = [torch.rand(n, generator=g, device="cuda").add_(0.1).mul_(size / 1.1).to(TYPES[dt]) for n in lengths]
    want = exact_norm(ts, "l2")
    out = [torch.empty_like(t) for t in ts]
    op = GradientNorm(ts, out=out)
    limit = float(torch.tensor(0.25 * want if want < 1e38 else 3e38))
    tol = SUM_TOL + 2.0 ** -23
    for got in (op.norm(), op.clip(limit)):
        if want < 3e38:
            assert abs(float(got) - want) <= tol * want + 2.0 ** -149
        else:
            assert float(got) == math.inf, "the float32 of a norm above its range"
    info = op.status()
    assert abs(info.norm - want) <= tol * want and abs(info.coef - limit / want) <= tol * info.coef and info.nonfinite == 0
    u = UNIT[TYPES[dt]]
    for t, o in zip(ts, out):
        x = t.double() * (limit / want)
        assert bool(((o.double() - x).abs() <= (u + tol + 2.0 ** -21) * x.abs() + (2.0 ** -149 if dt == "f32" else 2.0 ** -133)).all())
    op.close()


@gpu
@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
@pytest.mark.parametrize("n", [5000, 3_000_001])
def test_values_of_all_sizes_and_zeros_together(n, kind):
    """One huge value among tiny ones and zeros, and tiny ones among zeros; sums of magnitudes above float32's range."""
    for many, few in ((0.0, 1e-30), (1e-30, 1e25), (0.0, 1e25), (1e-25, 1.0), (3e38, 1e-30)):
        t = torch.full((n,), many, device="cuda")
        t[[1, n // 2, n - 1]] = few
        op = GradientNorm([t], out=[torch.empty_like(t)], kind=kind)
        want = exact_norm([t], kind)
        op.clip(1.0)
        info = op.status()
        assert abs(info.norm - want) <= SUM_TOL * want and info.nonfinite == 0
        assert abs(info.coef - min(1.0, 1.0 / want)) <= 2.0 ** -16 * info.coef
        op.close()


@gpu
@pytest.mark.parametrize("n", [5003, 3_000_001], ids=["one launch", "two launches"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_limit_far_below_the_norm(dt, n):
    """The factor is below float32's normal range (3e-43 here, 8 bits of one); the scaled values are not."""
    g = torch.Generator(device="cuda").manual_seed(6)
    for lead in (0, 1):
        t = torch.rand(n + lead, generator=g, device="cuda").add_(0.1).mul_(2e38).to(TYPES[dt])[lead:]
        want = exact_norm([t], "l2")
        limit = float(torch.tensor(3e-43 * want))
        out = torch.empty_like(t)
        ops = [GradientNorm([t], out=[out]), GradientNorm([t.clone()])]
        ops[0].clip(limit)
        x = t.double() * (limit / want)
        u = UNIT[TYPES[dt]]
        assert bool(((out.double() - x).abs() <= (u + SUM_TOL + 2.0 ** -21) * x.abs()).all())
        ops[1].clip(limit)
        assert torch.equal(ops[1]._tensors[0], out)
        [op.close() for op in ops]


@gpu
def test_equal_inputs_give_equal_bits_and_new_addresses_are_used():
    ts = tensors([100_003, 17, 900_000], [torch.bfloat16, torch.float32], seed=3)
    op = GradientNorm(ts)
    first = float(op.norm())
    assert all(float(op.norm()) == first for _ in range(50))
    moved = [t.clone() for t in ts]
    ts[0].zero_()
    op.bind(moved)
    assert float(op.norm()) == first
    with pytest.raises(ScarError):
        op.bind(moved[:-1])
    with pytest.raises(ScarError):
        op.bind([m[:-1] for m in moved])
    op.bind(moved)
    op.clip(first / 2)
    assert abs(float(op.norm()) - first / 2) <= 2e-3 * first
    op.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_new_addresses_that_begin_elsewhere(dt):
    """Tensors of whole pieces on 16-byte boundaries are later bound to places between two: each is cut into a piece more."""
    lengths = [16384 // torch.empty(0, dtype=TYPES[dt]).element_size()] * 300
    ts = tensors(lengths, [TYPES[dt]], seed=9)
    out = [torch.empty_like(t) for t in ts]
    op = GradientNorm(ts, out=out)
    first = float(op.clip(1.0))
    moved = tensors(lengths, [TYPES[dt]], seed=9, lead=(1,))  # other values, too
    place = [torch.full((n + 3,), 7.0, dtype=TYPES[dt], device="cuda") for n in lengths]
    op.bind(moved, out=[p[1:-2] for p in place])
    want = exact_norm(moved, "l2")
    got = float(op.clip(want / 2))
    assert abs(got - want) <= (SUM_TOL + 2.0 ** -23) * want and got != first
    u = UNIT[TYPES[dt]]
    for m, p in zip(moved, place):
        x = m.double() / 2
        assert bool(((p[1:-2].double() - x).abs() <= (u + SUM_TOL + 2.0 ** -21) * x.abs() + 2.0 ** -24).all())
        assert float(p[0]) == 7.0 and bool((p[-2:] == 7.0).all())
    op.bind(ts, out=out)
    assert float(op.clip(1.0)) == first
    op.close()


@gpu
def test_a_call_after_a_refused_bind():
    """The handle goes on with the tensors it had, which nobody else holds any more."""
    ts = tensors([100_003, 17], [torch.float32], seed=3)
    want = exact_norm(ts, "l2")
    op = GradientNorm(ts, kind="l2")
    del ts
    for bad in ([100_003], [100_003, 18], [100_002, 17]):
        with pytest.raises(ScarError):
            op.bind(tensors(bad, [torch.float32], seed=4))
    with pytest.raises(ScarError):
        op.bind(tensors([100_003, 17], [torch.bfloat16, torch.float32], seed=4))
    fresh = [torch.full((100_003,), 3.0, device="cuda") for _ in range(8)]  # would lie where freed tensors were
    assert abs(float(op.clip(want / 2)) - want) <= (SUM_TOL + 2.0 ** -23) * want
    assert all(bool((f == 3.0).all()) for f in fresh)
    assert abs(exact_norm(op._tensors, "l2") - want / 2) <= (SUM_TOL + 2.0 ** -20) * want
    op.close()


@gpu
def test_another_stream_and_a_captured_graph():
    ts = tensors([200_000, 11], [torch.float32], seed=4)
    out = [torch.empty_like(t) for t in ts]
    side = torch.cuda.Stream()
    op = GradientNorm(ts, out=out)
    want = float(op.clip(1.0))
    ref = [o.clone() for o in out]
    with torch.cuda.stream(side):
        for t in ts:
            t.mul_(2.0)
        got = op.clip(1.0)
        twice = got * 1
    side.synchronize()
    assert float(twice) == 2 * want
    assert all(torch.allclose(o, r, rtol=1e-6) for o, r in zip(out, ref))
    torch.cuda.synchronize()
    mine = GradientNorm(ts, out=out, stream=side)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mine.clip(1.0)
        for o in out:
            o.zero_()
        graph.replay()
    side.synchronize()
    assert all(torch.allclose(o, r, rtol=1e-6) for o, r in zip(out, ref))
    op.close()
    mine.close()


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("pieces", [3, 700], ids=["one launch", "two launches"])
def test_a_captured_call_follows_new_addresses(dt, pieces):
    """A graph holds a call's launches; bind then gives tensors that begin between two 16-byte boundaries, and others again."""
    size = torch.empty(0, dtype=TYPES[dt]).element_size()
    lengths = [16384 // size * pieces, 16384 // size, 5, 2 * 16384 // size - 1]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ts = tensors(lengths, [TYPES[dt]], seed=3)
        op = GradientNorm(ts, stream=side)
        norm = op.norm()  # the first call of the kernels is not a captured one
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norm = op.clip(1.0)
        for seed, lead in ((4, (1, 2, 3, 0)), (5, (0,)), (6, (7, 0, 1, 5))):
            moved = tensors(lengths, [TYPES[dt]], seed=seed, lead=lead)
            keep = [m.clone() for m in moved]
            side.synchronize()
            op.bind(moved)
            graph.replay()
            want = exact_norm(keep, "l2")
            assert abs(float(norm) - want) <= (SUM_TOL + 2.0 ** -23) * want
            for m, k in zip(moved, keep):
                x = k.double() / want
                tiny = 2.0 ** -24 if dt == "f16" else 0.0
                assert bool(((m.double() - x).abs() <= (UNIT[TYPES[dt]] + SUM_TOL + 2.0 ** -21) * x.abs() + tiny).all())
    side.synchronize()
    op.close()


@gpu
@pytest.mark.parametrize("kind", ["l2", "l1", "max"])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", ["one element", "zeros among them", "around a vector", "around a piece", "as many pieces as are resident", "hundreds of short ones"])
def test_a_wait_that_runs_out_changes_no_bit(name, dt, kind):
    """The CTAs of a clipping in one launch give up their wait at once: the last of them finishes the call alone, and the
    call after it finds everything as it was."""
    types = list(TYPES.values()) if dt == "mixed" else [TYPES[dt]]
    ts = tensors(LISTS[name], types, seed=5, lead=(0, 1, 3, 8), scale=1e-2)
    place = tensors(LISTS[name], types, seed=5, lead=(0, 1, 3, 8), scale=1e-2)  # the bits depend on the addresses modulo 16
    out = [torch.full_like(t, 7.0) for t in ts]
    want = [torch.empty_like(t) for t in ts]
    op, inp, ref = GradientNorm(ts, out=out, kind=kind), GradientNorm(place, kind=kind), GradientNorm(ts, out=want, kind=kind)
    limit = 0.4 * exact_norm(ts, kind)
    norm = float(ref.clip(limit))
    for turn in range(3):
        for o in (op, inp):
            if turn != 1:
                api.scar_gnorm_selftest_arm_timeout(o.op)
        [o.fill_(7.0) for o in out]
        [p.copy_(t) for p, t in zip(place, ts)]
        assert float(op.clip(limit)) == norm and float(inp.clip(limit)) == norm
        for o in (op, inp):
            assert (o.status().norm, o.status().coef) == (ref.status().norm, ref.status().coef)
            assert api.scar_gnorm_finished_alone(o.op) == (1, 1, 2)[turn]
        assert all(torch.equal(a, w) and torch.equal(p, w) for a, p, w in zip(out, place, want))
    assert api.scar_gnorm_finished_alone(ref.op) == 0
    [o.close() for o in (op, inp, ref)]


@gpu
def test_a_clipping_in_one_launch_beside_a_busy_gpu():
    """Other streams hold the multiprocessors while short lists are clipped: whichever way a call ends, its bits are the same."""
    ts = tensors([4096 * 500, 100_003], [torch.float32], seed=8)
    out = [torch.empty_like(t) for t in ts]
    op = GradientNorm(ts, out=out)
    norm = float(op.clip(1.0))
    want = [o.clone() for o in out]
    sides, a = [torch.cuda.Stream() for _ in range(2)], torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    for _ in range(10):
        for s in sides:
            with torch.cuda.stream(s):
                a @ a
        [o.zero_() for o in out]
        assert float(op.clip(1.0)) == norm and all(torch.equal(o, w) for o, w in zip(out, want))
    torch.cuda.synchronize()
    op.close()


@gpu
def test_refusals():
    t = torch.ones(8, device="cuda")
    with pytest.raises(TypeError):
        GradientNorm([t.int()])
    with pytest.raises(ValueError):
        GradientNorm([torch.ones(4, 4, device="cuda").T[1:]])
    with pytest.raises(ValueError):
        GradientNorm([t], out=[t[:4]])
    with pytest.raises(ValueError):
        GradientNorm([torch.ones(8)])
    op = GradientNorm([t])
    for bad in (-1.0, float("nan")):
        with pytest.raises(ScarError):
            op.clip(bad)
    with pytest.raises(ScarError):
        op.status()
    torch.cuda.synchronize()
    assert bool((t == 1).all())
    op.close()


@gpu
def test_a_norm_off_its_boundary_is_refused():
    t = torch.ones(8, device="cuda")
    op = GradientNorm([t])
    lib, room = api.load_library(), torch.full((4,), 3.0, device="cuda")
    for by in (1, 2, 3, 6):
        assert lib.scar_gnorm_norm(op.op, room.data_ptr() + by) == -1
        assert lib.scar_gnorm_clip(op.op, 1.0, room.data_ptr() + by) == -1
    assert api.scar_gnorm_launch_count(op.op) == 0
    torch.cuda.synchronize()
    assert bool((room == 3.0).all()) and bool((t == 1.0).all())
    op.close()


def test_arguments_are_checked_before_any_device_work():
    _build.build()
    lib = api.load_library()
    op = C.c_void_p(5)
    one = (api.scar_tensor * 1)()
    one[0].d_data, one[0].n_elems, one[0].dtype = 0x1000, 8, api.SCAR_F32
    assert lib.scar_gnorm_init(None, one, 1, 0, None) == -1
    assert lib.scar_gnorm_init(C.byref(op), None, 1, 0, None) == -1 and op.value is None
    assert lib.scar_gnorm_init(C.byref(op), one, 1, 3, None) == -1
    for field, value in (("dtype", api.SCAR_I32), ("dtype", 7), ("d_data", 0x1002), ("d_out", 0x1002), ("d_data", None)):
        t = (api.scar_tensor * 1)()
        t[0].d_data, t[0].n_elems, t[0].dtype = 0x1000, 8, api.SCAR_F32
        setattr(t[0], field, value)
        assert lib.scar_gnorm_init(C.byref(op), t, 1, 0, None) == -1, field
    t = (api.scar_tensor * 1)()
    t[0].d_data, t[0].n_elems, t[0].dtype = 0x1000, 1 << 48, api.SCAR_F32
    assert lib.scar_gnorm_init(C.byref(op), t, 1, 0, None) == -2
    assert lib.scar_gnorm_norm(None, None) == -1 and lib.scar_gnorm_clip(None, 1.0, None) == -1
    assert lib.scar_gnorm_bind(None, None, 0) == -1 and lib.scar_gnorm_status(None, None) == -1
    assert lib.scar_gnorm_destroy(None) == -1 and lib.scar_gnorm_launch_count(None) == 0


def test_the_calls_about_a_wait_check_their_arguments():
    _build.build()
    lib = api.load_library()
    assert lib.scar_gnorm_finished_alone(None, None) == -1 and lib.scar_gnorm_selftest_arm_timeout(None) == -1
