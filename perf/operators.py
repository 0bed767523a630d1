"""Cases for the operators of a training step: the linear softmax cross entropy with its gradient, and the global
gradient norm with clipping.

``own`` chooses between the library's calls and the same operators in elementary torch operations (32 bits throughout,
rounded once at the end).
"""

import math

import torch

own = False

IGNORE = -100
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the smallest training step worth a GPU (a tiny classifier head): launch latency counts
        {"name": "xent grad small", "op": "xent_grad", "dtype": "bf16", "tokens": 48, "classes": 4096, "dim": 512, "ignored": 0.0},
        # the repository's multinomial logistic regression: 1000 classes, 100,000 features, one minibatch in float32
        {"name": "xent grad mlr", "op": "xent_grad", "dtype": "f32", "tokens": 512, "classes": 1000, "dim": 100000, "ignored": 0.0},
        # an ordinary language model step: a micro-batch of 4096 tokens, some of them padding
        {"name": "xent grad ordinary", "op": "xent_grad", "dtype": "bf16", "tokens": 4096, "classes": 32000, "dim": 2048, "ignored": 0.1},
        # sizes that divide by nothing, packed sequences with the prompts left out of the loss
        {"name": "xent grad ragged", "op": "xent_grad", "dtype": "f16", "tokens": 1537, "classes": 50001, "dim": 1001, "ignored": 0.4},
        # the same step for a model trained in float32
        {"name": "xent grad float32", "op": "xent_grad", "dtype": "f32", "tokens": 2000, "classes": 10007, "dim": 768, "ignored": 0.1},
        # a large vocabulary and a wide model: the products are everything
        {"name": "xent grad large", "op": "xent_grad", "dtype": "bf16", "tokens": 8192, "classes": 128000, "dim": 4096, "ignored": 0.0},
        # evaluation (perplexity): the loss of every token, no gradient
        {"name": "xent loss eval", "op": "xent_loss", "dtype": "bf16", "tokens": 2048, "classes": 128000, "dim": 4096, "ignored": 0.1},
        # scoring one token: reading the weights is everything
        {"name": "xent loss one token", "op": "xent_loss", "dtype": "bf16", "tokens": 1, "classes": 128000, "dim": 4096, "ignored": 0.0},
        # one small flat gradient (the 2^20 parameters of the repository's tiny set): launch latency counts
        {"name": "clip tiny", "op": "clip", "dtype": "f32", "tensors": 1, "elems": 1 << 20, "clipped": True},
        # the norm alone, logged every step, of a gradient of the logistic regression's size
        {"name": "norm mlr", "op": "norm", "dtype": "f32", "tensors": 2, "elems": 100_001_000, "clipped": True},
        # the tensors of a network of a billion parameters in 16 bits
        {"name": "clip large", "op": "clip", "dtype": "bf16", "tensors": 290, "elems": 1_000_000_000, "clipped": True},
        # many tensors of all lengths and types, at odd places, a step whose norm is below the limit
        {"name": "clip ragged", "op": "clip", "dtype": "mixed", "tensors": 1200, "elems": 30_000_019, "clipped": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.6:
        op = "xent_loss" if rng.random() < 0.25 else "xent_grad"
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        while True:
            tokens, classes, dim = _log(rng, 1, 8192), _log(rng, 200, 128000), _log(rng, 64, 4096)
            if dtype == "f32" and rng.random() < 0.3:  # few classes, very many features
                classes, dim = _log(rng, 10, 2000), _log(rng, 4096, 100000)
            if rng.random() < 0.6:  # model widths are mostly multiples of 64
                dim = max(64, dim // 64 * 64)
            if tokens * classes * dim <= 8192 * 128000 * 4096 // 2 and dim != 3072:
                break
        return {"op": op, "dtype": dtype, "tokens": tokens, "classes": classes, "dim": dim,
                "ignored": rng.choice([0.0, 0.1, 0.5])}
    tensors = _log(rng, 1, 1200)
    return {"op": rng.choice(["norm", "clip", "clip"]), "dtype": rng.choice(["f32", "bf16", "f16", "mixed"]),
            "tensors": tensors, "elems": max(4 * tensors, _log(rng, 10_000, 500_000_000)), "clipped": rng.random() < 0.7}


def _kept(case):
    """Rows that count in the loss."""
    return case["tokens"] - int(case["tokens"] * case["ignored"])


def _lengths(case):
    """Lengths of the tensors: a few large ones, many small ones, odd ones among them; their sum is `elems`."""
    n, total = case["tensors"], case["elems"]
    if n == 1:
        return [total]
    weight = [math.exp(4.0 * math.cos(2.4 * i)) for i in range(n)]  # spread over a factor of 3000
    scale = (total - n) / sum(weight)
    got = [1 + int(scale * x) for x in weight]
    got[0] += total - sum(got)
    return got


def _types(case):
    if case["dtype"] != "mixed":
        return [case["dtype"]] * case["tensors"]
    return [("f32", "bf16", "f16")[i % 3] for i in range(case["tensors"])]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"].startswith("xent"):
        T, V, D, dt = case["tokens"], case["classes"], case["dim"], DTYPES[case["dtype"]]
        # logits of spread 1.5, the label's about 4 above the rest, as in a model that has learned something
        w = torch.randn(V, D, generator=g, device="cuda").mul_(1.5 / math.sqrt(D))
        labels = torch.randint(0, V, (T,), generator=g, device="cuda")
        h = torch.randn(T, D, generator=g, device="cuda").add_(w[labels], alpha=4 / 2.25).to(dt)
        w = w.to(dt)
        labels[torch.randperm(T, generator=g, device="cuda")[: int(T * case["ignored"])]] = IGNORE
        state = {"case": case, "h": h, "w": w, "labels": labels}
        if own:
            from paper_1810_07354_b200 import LinearCrossEntropy

            state["op"] = LinearCrossEntropy(T, V, D, dt, ignore_label=IGNORE)
        return state
    lengths, types = _lengths(case), _types(case)
    flat, out, grads, outs, norm2 = {}, {}, [None] * len(lengths), [None] * len(lengths), 0.0
    for t in sorted(set(types)):
        mine = [i for i, x in enumerate(types) if x == t]
        n = sum(lengths[i] for i in mine)
        flat[t] = torch.randn(n, generator=g, device="cuda").mul_(1e-2).to(DTYPES[t])
        out[t] = torch.empty_like(flat[t])
        norm2 += 1e-4 * n
        at = 0
        for i in mine:  # tensors lie one behind the other: odd lengths put those that follow at odd places
            grads[i], outs[i] = flat[t][at: at + lengths[i]], out[t][at: at + lengths[i]]
            at += lengths[i]
    state = {"case": case, "grads": grads, "outs": outs, "out": out,
             "max_norm": math.sqrt(norm2) * (0.3 if case["clipped"] else 2.0)}
    if own:
        from paper_1810_07354_b200 import GradientNorm

        state["op"] = GradientNorm(grads, out=outs)
    return state


def _xent_plain(h, w, labels, with_grad):
    h, w = h.float(), w.float()
    z = h @ w.T
    kept = labels != IGNORE
    at = labels.clamp(min=0)[:, None]
    top = z.max(dim=1, keepdim=True).values
    lse = top + (z - top).exp_().sum(dim=1, keepdim=True).log_()
    row_loss = torch.where(kept, (lse - z.gather(1, at))[:, 0], 0.0)
    n = kept.sum().clamp(min=1)
    loss = row_loss.sum() / n
    if not with_grad:
        return loss, row_loss
    dz = z.sub_(lse).exp_()
    dz.scatter_add_(1, at, torch.full_like(at, -1, dtype=dz.dtype))
    dz.mul_((kept / n)[:, None])
    return loss, row_loss, dz @ w, dz.T @ h


def run(state):
    case = state["case"]
    if case["op"].startswith("xent"):
        h, w, labels = state["h"], state["w"], state["labels"]
        with_grad = case["op"] == "xent_grad"
        if own:
            got = (state["op"].loss_and_grad if with_grad else state["op"].loss)(h, w, labels)
        else:
            got = _xent_plain(h, w, labels, with_grad)
        said = {"loss": got[0], "row_loss": got[1]}
        if with_grad:
            said |= {"dh": got[2].to(h.dtype), "dw": got[3].to(w.dtype)}
        return said
    grads, outs = state["grads"], state["outs"]
    if own:
        norm = state["op"].norm() if case["op"] == "norm" else state["op"].clip(state["max_norm"])
    else:
        norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
        if case["op"] == "clip":
            coef = (state["max_norm"] / norm).clamp(max=1.0)
            [torch.mul(g.float(), coef, out=o) for g, o in zip(grads, outs)]
    return {"norm": norm} if case["op"] == "norm" else {"norm": norm, **state["out"]}


def work(case):
    if case["op"].startswith("xent"):
        T, V, D, b, n = case["tokens"], case["classes"], case["dim"], SIZE[case["dtype"]], _kept(case)
        read = (T * D + V * D) * b + 8 * T
        if case["op"] == "xent_loss":
            return {"bytes": read + 4 * T + 4, "flops": 2 * n * V * D}
        return {"bytes": read + (T * D + V * D) * b + 4 * T + 4, "flops": 6 * n * V * D}
    moved = sum(n * SIZE[t] for n, t in zip(_lengths(case), _types(case)))
    if case["op"] == "norm":
        return {"bytes": moved + 4, "flops": 2 * case["elems"]}
    return {"bytes": 2 * moved + 4, "flops": 3 * case["elems"]}


def exact(case, seed):
    """The definitions in 64 bits, a few hundred rows at a time."""
    state = prepare(case, seed)
    if case["op"].startswith("xent"):
        with_grad = case["op"] == "xent_grad"
        h, w, labels = state["h"], state["w"].double(), state["labels"]
        T, V = h.shape[0], w.shape[0]
        n = max(1, int((labels != IGNORE).sum()))
        row_loss = torch.zeros(T, dtype=torch.float64, device="cuda")
        dh = torch.zeros(h.shape, dtype=torch.float64, device="cuda") if with_grad else None
        dw = torch.zeros_like(w) if with_grad else None
        step = max(1, (1 << 28) // V)
        for a in range(0, T, step):
            rows = torch.nonzero(labels[a: a + step] != IGNORE)[:, 0] + a
            if rows.numel() == 0:
                continue
            x, y = h[rows].double(), labels[rows]
            logp = torch.log_softmax(x @ w.T, dim=1)
            row_loss[rows] = torch.nn.functional.nll_loss(logp, y, reduction="none")
            if with_grad:
                r = (logp.exp() - torch.nn.functional.one_hot(y, V)) / n
                dh[rows] = r @ w
                dw += r.T @ x
        said = {"loss": row_loss.sum() / n, "row_loss": row_loss}
        return said | ({"dh": dh, "dw": dw} if with_grad else {})
    norm = math.sqrt(sum(float(torch.dot(g.double(), g.double())) for g in state["grads"]))
    if case["op"] == "norm":
        return {"norm": torch.tensor(norm, dtype=torch.float64)}
    coef = min(1.0, state["max_norm"] / norm) if norm else 1.0
    # the tensors of one type lie one behind the other in one buffer, and so do the results
    types = _types(case)
    return {"norm": torch.tensor(norm, dtype=torch.float64),
            **{t: torch.cat([g.double() * coef for g, x in zip(state["grads"], types) if x == t]) for t in state["out"]}}
