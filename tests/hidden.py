"""Plain forms of the operators of a hidden layer, for the tests: numpy and 64-bit torch, written from the formulas."""

import numpy as np

UNITS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}  # half a step, relative


def unit(dtype) -> float:
    return UNITS[str(dtype).replace("torch.", "")]


def smallest(dtype) -> float:
    """Half the smallest step: what a rounding may take from a value near 0."""
    return {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}[str(dtype).replace("torch.", "")]


def philox(c, k):
    """Philox 4x32 with ten rounds on Python ints: counter of four words, key of two."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def cut_of(p: float) -> int:
    if p in (0.0, 1.0):
        return int(p * 65536)
    return min(65535, max(1, int(np.floor(p * 65536 + 0.5))))


def mask(rows: int, cols: int, p: float, seed: int, offset: int, first_row: int = 0) -> np.ndarray:
    """The scaled mask, float64, by the definition, all rows at once in 64-bit words."""
    m32 = np.uint64(0xFFFFFFFF)
    blocks = -(-cols // 8)
    shape = (rows, blocks)
    c = [np.broadcast_to(np.arange(blocks, dtype=np.uint64), shape),
         np.broadcast_to(np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None], shape),
         np.full(shape, offset & 0xFFFFFFFF, dtype=np.uint64), np.full(shape, offset >> 32 & 0xFFFFFFFF, dtype=np.uint64)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32 & 0xFFFFFFFF)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)  # below 2^64
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & m32, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & m32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & m32, (k[1] + np.uint64(0xBB67AE85)) & m32]
    bits = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(rows, blocks * 8)[:, :cols]
    cut = cut_of(p)
    return (bits >= np.uint64(cut)) * (0.0 if cut == 65536 else 65536.0 / (65536 - cut))


def close(got, want, tol, what):
    """Every value within its bound; one that lies more than half a step beyond the type's largest (the bound taken off) rounds to
    infinity, in every type."""
    import torch

    info = torch.finfo(got.dtype)
    over = want.abs() - tol > info.max * (1 + info.eps / 4)  # half a step of the largest value's binade is eps / 4 of its upper end
    off = (got.double() - want).abs()
    bad = torch.where(over, got.double() != want.sign() * float("inf"), ~(off <= tol))
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float((off / tol.clamp(min=1e-300)).max()):.3g} of the bound"
