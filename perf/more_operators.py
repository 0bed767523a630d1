"""Cases for the operators of a hidden layer: the linear map with bias, activation, dropout and residual in its epilogue
and its gradients; dropout from a counter-based generator whose mask is never stored; the norms before and after a
residual block, fused with the block's gate and residual scale, and their gradients.

``own`` chooses between the library's calls and the same operators in elementary torch operations (32 bits throughout,
rounded once at the end).
"""

import functools
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def listed():
    return [
        # one row through a wide layer (an answer's next token): reading the weights is everything
        {"name": "linear one row", "op": "linear", "dtype": "bf16", "rows": 1, "inner": 4096, "outer": 16384, "act": "silu", "p": 0.0, "residual": False, "pad": 0},
        # a batch of sixteen answers through the layer back, with the residual
        {"name": "linear few rows", "op": "linear", "dtype": "bf16", "rows": 16, "inner": 8192, "outer": 4096, "act": "identity", "p": 0.0, "residual": True, "pad": 0},
        # the smallest training step of a hidden layer: launch latency counts
        {"name": "linear train small", "op": "linear_train", "dtype": "bf16", "rows": 64, "inner": 512, "outer": 512, "act": "gelu", "p": 0.1, "residual": True, "pad": 0},
        # a hidden layer under the repository's logistic regression: its minibatch and features, in float32
        {"name": "linear train mlr", "op": "linear_train", "dtype": "f32", "rows": 512, "inner": 4096, "outer": 2048, "act": "gelu", "p": 0.1, "residual": False, "pad": 0},
        # sizes that divide by nothing, rows taken out of a wider buffer
        {"name": "linear train ragged", "op": "linear_train", "dtype": "f16", "rows": 1537, "inner": 1001, "outer": 2003, "act": "silu", "p": 0.25, "residual": True, "pad": 5},
        # an ordinary step of a wide model: the products are everything
        {"name": "linear train large", "op": "linear_train", "dtype": "bf16", "rows": 8192, "inner": 4096, "outer": 16384, "act": "gelu", "p": 0.1, "residual": False, "pad": 0},
        # dropout of one small activation (2^20 values): launch latency counts
        {"name": "dropout small", "op": "dropout", "dtype": "f32", "rows": 1024, "cols": 1024, "p": 0.1, "residual": False, "pad": 0},
        # embeddings' dropout and its gradient over odd rows
        {"name": "dropout train ragged", "op": "dropout_train", "dtype": "f16", "rows": 4099, "cols": 5003, "p": 0.3, "residual": False, "pad": 3},
        # a block's output dropped and added to the residual stream
        {"name": "dropout residual large", "op": "dropout", "dtype": "bf16", "rows": 16384, "cols": 8192, "p": 0.1, "residual": True, "pad": 0},
        # one row through the norms around a block
        {"name": "norm one row", "op": "norm", "dtype": "bf16", "rows": 1, "dim": 4096, "kind": "rms", "post": True, "pre": True, "group": 0, "pad": 0},
        # sequences of 500 tokens, each with a gate of its own, in float32 with means and biases
        {"name": "norm train ragged", "op": "norm_train", "dtype": "f32", "rows": 3001, "dim": 1537, "kind": "layer", "post": True, "pre": True, "group": 500, "pad": 1},
        # an ordinary step of a wide model: both norms, a gate for every value
        {"name": "norm train large", "op": "norm_train", "dtype": "bf16", "rows": 16384, "dim": 4096, "kind": "rms", "post": True, "pre": True, "group": 1, "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.6 else n  # widths are mostly multiples of 64


def draw(rng):
    what = rng.random()
    dtype, pad = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 0, 3, 8])
    if what < 0.5:
        train = rng.random() < 0.6
        while True:
            rows, inner, outer = _log(rng, 1, 8192), _width(rng, 16, 16384), _width(rng, 16, 16384)
            if rows * inner * outer <= 8192 * 4096 * 16384 // (16 if dtype == "f32" else 2):
                break
        # values at relu's corner are left to inference: a sign there is the rounding's, and with it a whole gradient
        act = rng.choice(["identity", "gelu", "silu"] if train else ["identity", "relu", "gelu", "silu"])
        return {"op": "linear_train" if train else "linear", "dtype": dtype, "rows": rows, "inner": inner, "outer": outer, "act": act,
                "p": rng.choice([0.0, 0.1, 0.5]) if train else 0.0, "residual": rng.random() < 0.5, "pad": pad}
    if what < 0.7:
        while True:
            rows, cols = _log(rng, 1, 32768), _width(rng, 16, 16384)
            if rows * cols <= 8192 * 8192:
                break
        return {"op": rng.choice(["dropout", "dropout_train"]), "dtype": dtype, "rows": rows, "cols": cols,
                "p": rng.choice([0.05, 0.1, 0.5, 0.9]), "residual": rng.random() < 0.5, "pad": pad}
    while True:
        rows, dim = _log(rng, 1, 32768), _width(rng, 16, 8192)
        if rows * dim <= 16384 * 4096 // 2:
            break
    post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
    return {"op": rng.choice(["norm", "norm_train"]), "dtype": dtype, "rows": rows, "dim": dim, "kind": rng.choice(["rms", "layer"]),
            "post": post, "pre": pre, "group": rng.choice([0, 1, min(rows, 7), min(rows, 300), rows]), "pad": pad}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, pad = DTYPES[case["dtype"]], case["pad"]

    def values(*shape, spread=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(spread).add_(mean).to(dt)

    def rows(n, d, spread=1.0, mean=0.0):  # with `pad`, rows of a wider buffer that begin behind its first columns
        return values(n, d + pad, spread=spread, mean=mean)[:, pad:]

    op, state = case["op"], {"case": case}
    if op.startswith("linear"):
        T, K, N = case["rows"], case["inner"], case["outer"]
        state |= {"x": rows(T, K), "w": values(N, K, spread=1 / math.sqrt(K)), "bias": values(N, spread=0.2),
                  "residual": rows(T, N) if case["residual"] else None}
        if op == "linear_train":
            state["dy"] = values(T, N, spread=0.1)
    elif op.startswith("dropout"):
        state |= {"x": rows(case["rows"], case["cols"]), "residual": values(case["rows"], case["cols"]) if case["residual"] else None}
        if op == "dropout_train":
            state["dy"] = values(case["rows"], case["cols"], spread=0.1)
    else:
        T, D, group = case["rows"], case["dim"], case["group"]
        layer = case["kind"] == "layer"
        scale = lambda on: values(D, spread=0.1, mean=1.0) if on else None  # noqa: E731
        shift = lambda on: values(D, spread=0.1) if on and layer else None  # noqa: E731
        state |= {"x": rows(T, D, spread=2.0), "f": rows(T, D, spread=0.5, mean=0.1), "alpha": 0.5,
                  "gate": values(-(-T // group), D, spread=0.3, mean=0.5) if group else None,
                  "w_post": scale(case["post"]), "b_post": shift(case["post"]), "w_pre": scale(case["pre"]), "b_pre": shift(case["pre"])}
        if op == "norm_train":
            state |= {"dy": values(T, D, spread=0.1), "dn": values(T, D, spread=0.1) if case["pre"] else None}
    if not op.startswith("norm"):
        state |= {"seed": 0x9E3779B97F4A7C15 * (seed + 1) % 2**63, "offset": (1 << 32) + 7 * seed + 5}
    if own:
        from paper_1810_07354_b200 import Dropout, LinearLayer, ResidualNorm

        if op.startswith("linear"):
            state["op"] = LinearLayer(T, K, N, dt, activation=case["act"], forward_only=op == "linear")
            state["mask"] = Dropout(case["p"], state["seed"]).mask(state["offset"]) if case["p"] else None
        elif op.startswith("dropout"):
            state["op"] = Dropout(case["p"], state["seed"])
        else:
            state["op"] = ResidualNorm(T, D, dt, kind=case["kind"], eps=EPS, forward_only=op == "norm")
    return state


def _round(key, words):
    """One round of Philox 4x32 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011)."""
    a, b = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57
    low = 0xFFFFFFFF
    return [(b >> 32 & low) ^ words[1] ^ key[0], b & low, (a >> 32 & low) ^ words[3] ^ key[1], a & low]


def _mask(rows, cols, p, seed, offset):
    """The mask over rows x cols, scaled: ten rounds for every eight columns of a row, 16 bits for each value."""
    low = 0xFFFFFFFF
    block = torch.arange(-(-cols // 8), device="cuda").expand(rows, -1)
    row = torch.arange(rows, device="cuda")[:, None].expand_as(block)
    keys = [((seed + i * 0x9E3779B9) & low, ((seed >> 32) + i * 0xBB67AE85) & low) for i in range(10)]
    start = [block, row, torch.full_like(block, offset & low), torch.full_like(block, offset >> 32 & low)]
    words = torch.stack(functools.reduce(lambda w, k: _round(k, w), keys, start), dim=2)
    bits = torch.stack([words & 0xFFFF, words >> 16], dim=3).reshape(rows, -1)[:, :cols]
    cut = _cut(p)
    return (bits >= cut).float() * (65536.0 / (65536 - cut))


def _cut(p):
    return min(65535, max(1, math.floor(p * 65536 + 0.5))) if 0 < p < 1 else 0


def _activation(z, act):
    """The activation and its derivative."""
    if act == "identity":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + (-z).exp())
        return z * s, s * (1 + z * (1 - s))
    cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    return z * cdf, cdf + z * (-0.5 * z * z).exp() / math.sqrt(2 * math.pi)


def _linear_plain(s):
    case = s["case"]
    x, w = s["x"].float(), s["w"].float()
    a, slope = _activation(x @ w.T + s["bias"].float(), case["act"])
    mask = _mask(*a.shape, case["p"], s["seed"], s["offset"]) if case["p"] else 1.0
    y = a * mask
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if case["op"] == "linear":
        return {"y": y}
    dz = s["dy"].float() * mask * slope
    return {"y": y, "dx": dz @ w, "dw": dz.T @ x, "dbias": dz.sum(dim=0)}


def _dropout_plain(s):
    case = s["case"]
    mask = _mask(*s["x"].shape, case["p"], s["seed"], s["offset"])
    y = s["x"].float() * mask
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y} if case["op"] == "dropout" else {"y": y, "dx": s["dy"].float() * mask}


def _normed(v, layer):
    """(v - mean) / deviation, and 1 / deviation."""
    if layer:
        v = v - v.mean(dim=1, keepdim=True)
    r = 1 / (v.square().mean(dim=1, keepdim=True) + EPS).sqrt()
    return v * r, r


def _norm_back(du, hat, r, layer):
    if layer:
        du = du - du.mean(dim=1, keepdim=True)
    return r * (du - hat * (du * hat).mean(dim=1, keepdim=True))


def _norm_plain(s):
    case, layer = s["case"], s["case"]["kind"] == "layer"
    x, f, alpha = s["x"].float(), s["f"].float(), s["alpha"]
    gate = None if s["gate"] is None else s["gate"].float().repeat_interleave(case["group"], dim=0)[: x.shape[0]]
    u = f
    if case["post"]:
        f_hat, f_r = _normed(f, layer)
        u = f_hat * s["w_post"].float() + (s["b_post"].float() if layer else 0)
    y = x + alpha * (u if gate is None else gate * u)
    said = {"y": y}
    if case["pre"]:
        # the norm is that of the values handed on
        y_hat, y_r = _normed(y.to(s["x"].dtype).float(), layer)
        said["n"] = y_hat * s["w_pre"].float() + (s["b_pre"].float() if layer else 0)
    if case["op"] == "norm":
        return said
    dx = s["dy"].float()
    if case["pre"]:
        dn = s["dn"].float()
        dx = dx + _norm_back(dn * s["w_pre"].float(), y_hat, y_r, layer)
        said["dw_pre"] = (dn * y_hat).sum(dim=0)
        if layer:
            said["db_pre"] = dn.sum(dim=0)
    said["dx"] = dx
    du = alpha * (dx if gate is None else dx * gate)
    if gate is not None:
        pad = s["gate"].shape[0] * case["group"] - x.shape[0]
        each = torch.cat([alpha * dx * u, torch.zeros(pad, x.shape[1], device="cuda")])
        said["dgate"] = each.view(s["gate"].shape[0], case["group"], -1).sum(dim=1)
    if case["post"]:
        said["dw_post"] = (du * f_hat).sum(dim=0)
        if layer:
            said["db_post"] = du.sum(dim=0)
        du = _norm_back(du * s["w_post"].float(), f_hat, f_r, layer)
    said["df"] = du
    return said


def run(state):
    case, op = state["case"], state["case"]["op"]
    if not own:
        plain = _linear_plain if op.startswith("linear") else _dropout_plain if op.startswith("dropout") else _norm_plain
        dt = state["x"].dtype
        return {k: v.to(dt) for k, v in sorted(plain(state).items())}
    if op.startswith("linear"):
        layer, x, w, mask = state["op"], state["x"], state["w"], state["mask"]
        if op == "linear":
            return {"y": layer.forward(x, w, bias=state["bias"], residual=state["residual"], dropout=mask)}
        y, slope = layer.forward_train(x, w, bias=state["bias"], residual=state["residual"], dropout=mask)
        dx, dw, dbias = layer.backward(state["dy"], x, w, slope, dropout=mask)
        return {"dbias": dbias, "dw": dw, "dx": dx, "y": y}
    if op.startswith("dropout"):
        drop, offset = state["op"], state["offset"]
        y = drop.forward(state["x"], offset, residual=state["residual"])
        return {"y": y} if op == "dropout" else {"dx": drop.backward(state["dy"], offset), "y": y}
    norm = state["op"]
    with_block = {k: state[k] for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")} | {"scale": state["alpha"], "rows_per_gate": case["group"] or 1}
    y, n = norm.forward(state["x"], state["f"], post=case["post"], pre=case["pre"], **with_block)
    said = {"y": y} | ({"n": n} if case["pre"] else {})
    if op == "norm_train":
        grads = norm.backward(state["dy"], state["dn"], y, state["f"], post=case["post"], pre=case["pre"], **with_block)
        said |= {k: v for k, v in grads.items() if v is not None}
    return dict(sorted(said.items()))


def work(case):
    b, op = SIZE[case["dtype"]], case["op"]
    if op.startswith("linear"):
        T, K, N = case["rows"], case["inner"], case["outer"]
        moved = T * K + N * K + N + T * N + (T * N if case["residual"] else 0)
        if op == "linear":
            return {"bytes": moved * b, "flops": 2 * T * K * N}
        return {"bytes": (moved + T * N + T * K + N * K + N) * b, "flops": 6 * T * K * N}
    if op.startswith("dropout"):
        n = case["rows"] * case["cols"]
        passes = 2 + (1 if case["residual"] else 0) + (2 if op == "dropout_train" else 0)
        return {"bytes": passes * n * b, "flops": (1 + (op == "dropout_train")) * 2 * n}
    T, D, G = case["rows"], case["dim"], -(-case["rows"] // case["group"]) if case["group"] else 0
    n, vectors = T * D, (case["post"] + case["pre"]) * (2 if case["kind"] == "layer" else 1) * D
    norms = case["post"] + case["pre"]
    moved, flops = 3 * n + G * D + vectors + (n if case["pre"] else 0), (3 + 5 * norms) * n
    if op == "norm_train":
        moved += 3 * n + G * D + vectors + (n if case["pre"] else 0)
        flops += (4 + 10 * norms) * n
    return {"bytes": moved * b, "flops": flops}


def exact(case, seed):
    """The definitions in 64 bits, their gradients by automatic differentiation."""

    def scaled_mask(rows, cols, p, seed, offset):
        """The scaled mask in 64 bits; the generator's products from 16-bit halves."""
        low, m16 = 0xFFFFFFFF, 0xFFFF

        def product(v, c):  # high and low word of v * c for 32-bit v and c
            p0, p1 = (v & m16) * c, (v >> 16) * c
            mid = p1 + (p0 >> 16)
            return mid >> 16, (mid & m16) << 16 | p0 & m16

        cut, step = _cut(p), max(1, (1 << 24) // max(1, cols))
        got = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
        for at in range(0, rows, step):
            n = min(step, rows - at)
            w0 = torch.arange(-(-cols // 8), device="cuda").repeat(n, 1)
            w1 = torch.arange(at, at + n, device="cuda")[:, None] + torch.zeros_like(w0)
            w2, w3 = torch.zeros_like(w0) + (offset & low), torch.zeros_like(w0) + (offset >> 32 & low)
            k0, k1 = seed & low, seed >> 32 & low
            for _ in range(10):
                (h0, l0), (h1, l1) = product(w0, 0xD2511F53), product(w2, 0xCD9E8D57)
                w0, w1, w2, w3 = h1 ^ w1 ^ k0, l1, h0 ^ w3 ^ k1, l0
                k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
            for j, word in enumerate((w0, w1, w2, w3)):
                for h in range(2):
                    at_col = got[at: at + n, 2 * j + h:: 8]
                    at_col.copy_((word >> 16 * h & m16)[:, : at_col.shape[1]] >= cut)
        return got.mul_(1.0 / (1.0 - cut / 65536.0))

    s = {k: v.double().requires_grad_() if torch.is_tensor(v) else v for k, v in prepare(case, seed).items()}
    op, dy = case["op"], s.get("dy")
    mask = scaled_mask(case["rows"], case.get("cols", case.get("outer")), case["p"], s["seed"], s["offset"]) if case.get("p") else 1.0
    if op.startswith("dropout"):
        y = s["x"] * mask + (0 if s["residual"] is None else s["residual"])
        want, names = [s["x"]], ["dx"]
        ends, grads = [y], [dy]
    elif op.startswith("linear"):
        z = torch.nn.functional.linear(s["x"], s["w"], s["bias"])
        a = {"identity": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]](z)
        y = a * mask + (0 if s["residual"] is None else s["residual"])
        want, names = [s["x"], s["w"], s["bias"]], ["dx", "dw", "dbias"]
        ends, grads = [y], [dy]
    else:
        def normed(v, w, b):
            if case["kind"] == "layer":
                return torch.nn.functional.layer_norm(v, v.shape[1:], w, b, EPS)
            return torch.nn.functional.rms_norm(v, v.shape[1:], w, EPS)

        u = normed(s["f"], s["w_post"], s["b_post"]) if case["post"] else s["f"]
        which = torch.arange(case["rows"], device="cuda") // max(1, case["group"])
        y = s["x"] + s["alpha"] * (u if s["gate"] is None else s["gate"][which] * u)
        ends, grads = [y], [dy]
        if case["pre"]:
            # of the values handed on, which are rounded: the rounding has the derivative of the identity
            kept = y + (y.detach().to(DTYPES[case["dtype"]]).double() - y.detach())
            n = normed(kept, s["w_pre"], s["b_pre"])
            ends, grads = [y, n], [dy, s.get("dn")]
        pairs = {"dx": s["x"], "df": s["f"], "dgate": s["gate"], "dw_post": s["w_post"], "db_post": s["b_post"], "dw_pre": s["w_pre"], "db_pre": s["b_pre"]}
        names, want = zip(*[(k, v) for k, v in pairs.items() if v is not None])
    said = {"y": y.detach()} | ({"n": ends[1].detach()} if len(ends) == 2 else {})
    if op.endswith("train"):
        said |= dict(zip(names, torch.autograd.grad(ends, want, [g.detach() for g in grads])))
    return dict(sorted(said.items()))
