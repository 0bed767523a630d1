"""Dropout against the definition: the mask bit for bit, the values within the roundings that the call makes."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from hidden import close, cut_of, mask, philox, smallest, unit  # noqa: E402
from paper_1810_07354_b200 import Dropout, LinearLayer  # noqa: E402

gpu = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def test_the_plain_generator_gives_the_published_words():
    """The known answers that the generator's authors publish for ten rounds."""
    assert philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_the_plain_mask_is_made_of_those_words():
    seed, offset, p = 0x123456789ABCDEF0, (7 << 32) + 9, 0.3
    m = mask(3, 21, p, seed, offset)
    for r in range(3):
        for c in range(21):
            w = philox([c // 8, r, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32])[c % 8 // 2]
            bits = w >> 16 if c % 2 else w & 0xFFFF
            assert (m[r, c] != 0) == (bits >= cut_of(p))
    assert m.max() == 65536 / (65536 - 19661)


def check(y, x, res, m, dt):
    """Product, sum and result are rounded once each: to float32, to float32, to the type."""
    m = torch.from_numpy(m).cuda().view(x.shape)
    want = torch.where(m == 0, 0.0, x.double() * m)
    tol = 2.0 ** -24 * want.abs() * 2
    if res is not None:
        want = want + res.double()
        tol = tol + 2.0 ** -24 * want.abs()
    close(y, want, tol + unit(dt) * want.abs() * (1 + 2.0 ** -20) + smallest(dt), "dropout")
    if res is None:
        assert bool(((y == 0) == ((m == 0) | (x == 0))).all()), "which values are dropped"


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,p", [
    (1, 1, 0, 0.5), (1, 7, 0, 0.5), (3, 8, 0, 0.1), (5, 9, 0, 0.25), (2, 255, 1, 0.9), (64, 256, 0, 0.1), (33, 257, 3, 0.5), (300, 1000, 0, 0.05),
    (17, 1024, 8, 0.3), (1000, 24, 0, 0.5), (129, 4099, 0, 0.2), (1, 100001, 0, 0.1), (50, 520, 4, 1e-7), (50, 520, 4, 1 - 1e-7),
])
def test_values(dt, rows, cols, pad, p):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    wide = torch.randn(rows, cols + pad, generator=g, device="cuda").to(TYPES[dt])
    x, res, seed, offset = wide[:, pad:], torch.randn(rows, cols, generator=g, device="cuda").to(TYPES[dt]), 2**63 + 12345, (1 << 35) + cols
    drop, m = Dropout(p, seed), mask(rows, cols, p, seed, offset)
    check(drop.forward(x, offset), x, None, m, x.dtype)
    check(drop.forward(x, offset, residual=res), x, res, m, x.dtype)
    check(drop.backward(res, offset), res, None, m, x.dtype)
    # in place, into rows of a wider buffer, whose other columns stay
    before = wide.clone()
    got = drop.forward(x, offset, residual=res, out=x)
    assert got.data_ptr() == x.data_ptr()
    check(x, before[:, pad:], res, m, x.dtype)
    assert torch.equal(wide[:, :pad], before[:, :pad])


@gpu
def test_far_offsets_and_long_buffers():
    """Rows beyond 2^32 bytes and elements, 64-bit seeds and offsets."""
    rows, cols = 70000, 65536  # 2^32 values and more
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    Dropout(0.5, 2**64 - 1).forward(x, 2**64 - 2, out=x)
    for r in (0, 65535, 65536, 69999):
        assert np.array_equal(x[r].double().cpu().numpy(), mask(1, cols, 0.5, 2**64 - 1, 2**64 - 2, r)[0])
    x = x.view(-1)[1:].view(-1)[: 69999 * 65536].view(69999, 65536)  # rows off every boundary
    y = Dropout(0.5, 5).forward(x, 1, out=x.fill_(1))
    for r in (0, 65536, 69998):
        assert np.array_equal(y[r].double().cpu().numpy(), mask(1, cols, 0.5, 5, 1, r)[0])


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
def test_ends_of_the_range_and_what_is_dropped(dt):
    x = torch.full((40, 100), float("nan"), device="cuda", dtype=TYPES[dt])
    x[::2] = float("inf")
    res = torch.randn(40, 100, device="cuda").to(TYPES[dt])
    assert torch.equal(Dropout(1.0).forward(x, residual=res), res) and bool((Dropout(1.0).forward(x) == 0).all())
    y = torch.randn(40, 100, device="cuda").to(TYPES[dt])
    assert torch.equal(Dropout(0.0).forward(y), y)
    for got in (Dropout(0.5, 3).forward(x), Dropout(0.5, 3).forward(x[:, 1:])):  # aligned and not
        m = torch.from_numpy(mask(40, got.shape[1], 0.5, 3, 0)).cuda() != 0
        assert bool((got[~m] == 0).all()) and bool((~got[m].isfinite()).all())
    assert Dropout(0.5).forward(x[:0]).shape == (0, 100) and Dropout(0.5).forward(x[:, :0]).shape == (40, 0)


@gpu
def test_any_number_of_dimensions():
    x = torch.randn(4, 6, 40, device="cuda")
    m = torch.from_numpy(mask(24, 40, 0.5, 1, 2)).cuda().view(4, 6, 40)
    for got in (Dropout(0.5, 1).forward(x, 2), Dropout(0.5, 1).forward(x.view(24, 40), 2).view(4, 6, 40)):
        assert torch.equal(got, (x * m).float())
    v = torch.randn(99, device="cuda")
    assert torch.equal(Dropout(0.5, 1).forward(v), (v * torch.from_numpy(mask(1, 99, 0.5, 1, 0)[0]).cuda()).float())
    for bad in (torch.randn(6, 4, device="cuda").t(), torch.randn(2, 5, 6, device="cuda")[:, ::2].transpose(0, 1)):
        with pytest.raises(ValueError):
            Dropout(0.5).forward(bad)


@gpu
def test_share_and_independence():
    """Of 2^22 values the kept share is within six standard deviations of 1 - p; masks of other offsets, seeds and rows agree
    where chance has it."""
    x = torch.ones(1024, 4096, device="cuda")
    for p in (0.1, 0.5, 0.9):
        kept = [Dropout(p, s).forward(x, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0), (1, 1 << 32))]
        n = x.numel()
        for k in kept:
            assert abs(float(k.double().mean()) - (1 - p)) <= 6 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17
        same = p * p + (1 - p) ** 2
        for other in kept[1:] + [kept[0].roll(1, 0), kept[0].roll(1, 1), kept[0].roll(8, 1)]:
            assert abs(float((kept[0] == other).double().mean()) - same) <= 6 * (same * (1 - same) / n) ** 0.5 + 2.0 ** -15


@gpu
def test_a_captured_call_takes_the_offset_of_its_replay():
    x, offset = torch.randn(64, 129, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    drop = Dropout(0.4, 9, stream=stream)
    with torch.cuda.stream(stream):
        y = drop.forward(x, offset)  # warm
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = drop.forward(x, offset)
    torch.cuda.synchronize()
    for at in (0, 5, 2**40, -1):
        offset.fill_(at)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, drop.forward(x, at if at >= 0 else 2**64 - 1))


@gpu
def test_another_stream_than_the_callers():
    """The handle's stream waits for what the caller's has under way, and the other way round."""
    drop, other = Dropout(0.5, 4, stream=torch.cuda.Stream()), torch.cuda.Stream()
    want = torch.from_numpy(mask(2048, 2048, 0.5, 4, 8)).cuda().float()
    with torch.cuda.stream(other):
        for _ in range(20):
            x = torch.zeros(2048, 2048, device="cuda")
            for _ in range(10):
                x = x + 0.5
            y = drop.forward(x, 8) * 2
            del x
            assert torch.equal(y, want * 10)


@gpu
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("T,N,K", [(70, 300, 64), (3, 1000, 2048), (600, 264, 40)])
def test_a_layer_has_the_same_mask(dt, T, N, K):
    x, w = torch.randn(T, K, device="cuda").to(TYPES[dt]), torch.randn(N, K, device="cuda").to(TYPES[dt])
    layer, drop = LinearLayer(T, K, N, TYPES[dt], activation="identity"), Dropout(0.3, 77)
    whole, dropped = layer.forward(x, w), layer.forward(x, w, dropout=drop.mask(6))
    m = torch.from_numpy(mask(T, N, 0.3, 77, 6)).cuda()
    assert bool((dropped[m == 0] == 0).all())
    kept = (whole.double() * m)[m != 0]
    # dropped rounds z m once, whole z: two roundings apart
    assert bool(((dropped.double()[m != 0] - kept).abs() <= (2 * unit(TYPES[dt]) + 2.0 ** -22) * kept.abs() * 1.01 + 2 * smallest(TYPES[dt])).all())
    layer.close()
