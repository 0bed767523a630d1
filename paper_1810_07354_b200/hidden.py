"""Hidden layers in front of a classifier, on the library's operators: the part of a network between its input and its
loss whose parameters a running checkpoint keeps (the paper's Section 5.1 partitions a network's parameters by layer or by
shard; its convolutional network ends in fully connected layers with activations between them).

    h = dropout(gelu(x w_in^T + b_in))
    for every block:   f = w2 dropout(gelu(w1 N(h; pre) + b1)) + b2,   h = h + scale gate N(f; post)
    n = N(h; pre)                                  N(v; w) = v / sqrt(mean v^2 + eps) w

All parameters lie in one float32 buffer and their gradients in another of the same layout, so that one
:class:`~paper_1810_07354_b200.ScarCheckpoint` holds them and one :class:`~paper_1810_07354_b200.GradientNorm` clips them.  The masks of a
step come from the seed and the step's number alone: a step that is taken again after a recovery drops the same values.
"""

from __future__ import annotations

import math

from . import api


class HiddenLayers:
    def __init__(self, features: int, hidden: int, blocks: int, batch: int, inner: int = 0, dropout: float = 0.1, scale: float = 1.0, seed: int = 0):
        import torch

        inner = inner or 2 * hidden
        shapes = {"w_in": (hidden, features), "b_in": (hidden,), "pre0": (hidden,)}
        for i in range(blocks):
            shapes |= {f"w1_{i}": (inner, hidden), f"b1_{i}": (inner,), f"w2_{i}": (hidden, inner), f"b2_{i}": (hidden,), f"post{i}": (hidden,),
                       f"gate{i}": (1, hidden), f"pre{i + 1}": (hidden,)}
        self.features, self.hidden, self.blocks, self.batch, self.scale = features, hidden, blocks, batch, scale
        self._shapes, size = shapes, sum(-(-math.prod(v) // 4) * 4 for v in shapes.values())
        self.place(torch.zeros(size, device="cuda"), torch.zeros(size, device="cuda"))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for name, v in self.p.items():
            if v.dim() == 2 and name[0] == "w":
                v.normal_(0.0, 1 / math.sqrt(v.shape[1]), generator=gen)
            elif name[0] != "b":
                v.fill_(1.0)
        f32 = torch.float32
        self.drop = api.Dropout(dropout, seed) if dropout else None
        self.first = api.LinearLayer(batch, features, hidden, f32, activation="gelu")
        self.up = api.LinearLayer(batch, hidden, inner, f32, activation="gelu")
        self.down = api.LinearLayer(batch, inner, hidden, f32, activation="identity")
        self.norm = api.ResidualNorm(batch, hidden, f32, kind="rms")

    def place(self, params, grads):
        """Takes parameters and gradients from these float32 buffers (of ``params.numel()`` values each) from now on."""
        at, self.p, self.g = 0, {}, {}
        for name, shape in self._shapes.items():  # each on a 16-byte boundary where the buffer is on one
            n = math.prod(shape)
            self.p[name], self.g[name] = params[at: at + n].view(shape), grads[at: at + n].view(shape)
            at += -(-n // 4) * 4
        self.params, self.grads = params, grads

    def _mask(self, step: int, which: int):
        return None if self.drop is None else self.drop.mask(step * (self.blocks + 1) + which)

    def _block(self, i: int):
        return dict(scale=self.scale, gate=self.p[f"gate{i}"], rows_per_gate=self.batch, w_post=self.p[f"post{i}"], w_pre=self.p[f"pre{i + 1}"])

    def forward(self, x, step: int):
        """The classifier's input ``n``; what backward needs is kept until then."""
        p = self.p
        h, slope = self.first.forward_train(x, p["w_in"], p["b_in"], dropout=self._mask(step, 0))
        _, n = self.norm.forward(h, w_pre=p["pre0"])
        self.kept = [(x, slope, h)]
        for i in range(self.blocks):
            a, slope = self.up.forward_train(n, p[f"w1_{i}"], p[f"b1_{i}"], dropout=self._mask(step, i + 1))
            f = self.down.forward(a, p[f"w2_{i}"], p[f"b2_{i}"])
            h, m = self.norm.forward(h, f, **self._block(i))
            self.kept.append((n, slope, a, f, h))
            n = m
        return n

    def backward(self, dn, step: int):
        """Fills the gradients from that of ``n``, with the step's number of the forward call."""
        p, g, dh = self.p, self.g, None
        for i in reversed(range(self.blocks)):
            n, slope, a, f, h = self.kept.pop()
            got = self.norm.backward(dh, dn, h, f, **self._block(i), out={"dgate": g[f"gate{i}"], "dw_post": g[f"post{i}"], "dw_pre": g[f"pre{i + 1}"]})
            da, _, _ = self.down.backward(got["df"], a, p[f"w2_{i}"], None, dw=g[f"w2_{i}"], dbias=g[f"b2_{i}"])
            dn, _, _ = self.up.backward(da, n, p[f"w1_{i}"], slope, dropout=self._mask(step, i + 1), dw=g[f"w1_{i}"], dbias=g[f"b1_{i}"])
            dh = got["dx"]
        x, slope, h = self.kept.pop()
        dh = self.norm.backward(dh, dn, h, w_pre=p["pre0"], out={"dw_pre": g["pre0"]})["dx"]
        self.first.backward(dh, x, p["w_in"], slope, dropout=self._mask(step, 0), dw=g["w_in"], dbias=g["b_in"], need_dx=False)

    def status(self) -> None:
        """Waits; raises if a wait inside a kernel of the calls since the last status gave up: parameters trained on since then are not to
        be saved."""
        for op in (self.first, self.up, self.down, self.norm):
            op.status()

    def launches(self) -> int:
        return sum(api.scar_linear_launch_count(op.op) for op in (self.first, self.up, self.down)) + api.scar_resnorm_launch_count(self.norm.op)

    def close(self):
        for op in (self.first, self.up, self.down, self.norm):
            op.close()
