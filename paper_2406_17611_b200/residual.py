"""Residual feed-forward blocks between the graph layers, with 8-bit products and clipped steps.

Stacks deeper than the paper's three layers train with a residual stream.  Every hidden graph layer l is followed by a
block that works on each node by itself; with s the stream, x the layer's normalised input, N the RMS norm with a gain:

    y  = layer_l(x)                              varco_layer_fwd: exchange, aggregation, transform, ReLU
    s1 = s + y,           x1 = N(s1)             varco_norm_fwd (bf16 / fp32 and 8 bits in one pass)
    u  = relu(x1 W1^T + b1)                      varco_fp8_product, its output again in 8 bits
    s2 = s1 + u W2^T + b2,  x' = N(s2)           varco_fp8_product, varco_norm_fwd

x' is the next layer's input; where a layer changes the width the stream begins anew (s = 0).  The backward pass takes
the gradients in 8 bits through both products (varco_fp8_product on the transposed weights) and keeps the weight
gradients in the activation type (varco_weight_grad).  The blocks see no partition boundary: only the graph layers
communicate, and their halo bytes are what they are without the blocks.
"""
from __future__ import annotations

import numpy as np

from . import binding as vb
from .train import Trainer


class FeedForward:
    """One block: weights W1 [hidden x width], b1, W2 [width x hidden], b2 and the gains of its two norms, fp32 on the
    device; their 8-bit forms are made by refresh(), which has to follow every change of the weights."""

    NAMES = ("W1", "b1", "W2", "b2", "gain1", "gain2")

    def __init__(self, width, hidden, arrays, dtype, workspace, device):
        import torch
        self.width, self.hidden, self.dtype, self.ws = int(width), int(hidden), dtype, workspace
        shapes = {"W1": (hidden, width), "b1": (hidden,), "W2": (width, hidden), "b2": (width,), "gain1": (width,), "gain2": (width,)}
        for name in self.NAMES:
            a = np.ascontiguousarray(arrays[name], dtype=np.float32)
            if a.shape != shapes[name]:
                raise ValueError("%s has shape %s, not %s" % (name, a.shape, shapes[name]))
            setattr(self, name, torch.from_numpy(a).to(device))
        self.grad_ws = vb.varco_weight_grad_workspace(max(width, hidden), max(width, hidden), device)
        self.refresh()

    @staticmethod
    def init(width, hidden, seed):
        """Glorot-uniform weights, zero biases, unit gains."""
        rng = np.random.default_rng(seed)
        b = np.sqrt(6.0 / (width + hidden))
        return {"W1": rng.uniform(-b, b, (hidden, width)), "b1": np.zeros(hidden), "W2": rng.uniform(-b, b, (width, hidden)),
                "b2": np.zeros(width), "gain1": np.ones(width), "gain2": np.ones(width)}

    def parameters(self):
        return [getattr(self, n) for n in self.NAMES]

    def refresh(self):
        self.q1, self.q2 = vb.varco_quantize_weight(self.W1), vb.varco_quantize_weight(self.W2)

    def forward(self, y, stream=None):
        """y: output rows of the graph layer; stream: rows of the residual stream or None.  Returns (x', new stream)."""
        F, dt = self.width, self.dtype
        n1 = vb.varco_norm_fwd(y, F, gain=self.gain1, residual=stream, quantize=True)
        self.s1 = y if stream is None else n1.H
        self.x1, self.rstd1 = n1.Y, n1.rstd
        u = vb.varco_fp8_product(n1.Y8, n1.scales, self.q1.data, self.q1.scales, F, bias=self.b1, relu=True, dtype=dt, quantize=True,
                                 workspace=self.ws)
        self.u = u.Y
        v = vb.varco_fp8_product(u.Y8, u.scales, self.q2.data, self.q2.scales, self.hidden, bias=self.b2, dtype=dt, workspace=self.ws)
        n2 = vb.varco_norm_fwd(v.Y, F, gain=self.gain2, residual=self.s1)
        self.s2, self.rstd2 = n2.H, n2.rstd
        return n2.Y, n2.H

    def backward(self, dx, dstream=None):
        """dx: gradient of x'; dstream: gradient that reaches the new stream past x' (None for the last block).  Returns
        (gradient of y, which is that of the incoming stream too; gradients in the order of parameters())."""
        F, dt = self.width, self.dtype
        d2 = vb.varco_norm_bwd(dx, self.s2, self.rstd2, F, gain=self.gain2, residual_grad=dstream, quantize=True, workspace=self.ws)
        dz = vb.varco_fp8_product(d2.dX8, d2.scales, self.q2.transposed, self.q2.scales.t(), F, mask=self.u, dtype=dt, quantize=True,
                                  workspace=self.ws)
        dW2, db2 = vb.varco_weight_grad(d2.dX, F, self.u, self.hidden, self.grad_ws)
        dx1 = vb.varco_fp8_product(dz.Y8, dz.scales, self.q1.transposed, self.q1.scales.t(), self.hidden, dtype=dt, workspace=self.ws)
        dW1, db1 = vb.varco_weight_grad(dz.Y, self.hidden, self.x1, F, self.grad_ws)
        d1 = vb.varco_norm_bwd(dx1.Y, self.s1, self.rstd1, F, gain=self.gain1, residual_grad=d2.dX, workspace=self.ws)
        return d1.dX, [dW1, db1, dW2, db2, d1.dgain, d2.dgain]


class ResidualTrainer(Trainer):
    """Trainer whose hidden layers are followed by feed-forward blocks and whose steps are clipped: the norm over the
    averaged gradients of all weights (graph layers and blocks) is kept below max_norm.  `hidden`: the blocks' inner width;
    `blocks`: their initial arrays, one dict of FeedForward.init's form for every hidden layer (drawn from `seed` if None).
    bf16 layers read bf16 copies, the blocks' products 8-bit forms; the step renews both, and refresh() has to follow every other
    change of the weights (a checkpoint that is read into them)."""

    def __init__(self, plan, widths, weights, bf16, hidden, max_norm=1.0, blocks=None, seed=0, device="cuda:0"):
        super().__init__(plan, widths, weights, bf16, device)
        torch = self.torch
        if not max_norm > 0:
            raise ValueError("max_norm must be positive")
        self.max_norm = float(max_norm)
        inner = self.widths[1:-1]
        self.op_ws = vb.varco_ops_workspace(max(inner + [1]), device)
        if blocks is None:
            blocks = [FeedForward.init(w, hidden, seed + l) for l, w in enumerate(inner)]
        if len(blocks) != len(inner):
            raise ValueError("one block for every hidden layer: %d, not %d" % (len(inner), len(blocks)))
        self.blocks = [FeedForward(w, hidden, b, self.dt, self.op_ws, device) for w, b in zip(inner, blocks)]
        # what the layers read: the weights themselves, or the bf16 copies of the matrices
        self.low = [[None if w is None else w.to(torch.bfloat16) if bf16 and w.dim() == 2 else None for w in layer] for layer in self.W]

    def refresh(self):
        """The bf16 copies of the layers' weights and the 8-bit forms of the blocks' are made from the weights again."""
        for layer, low in zip(self.W, self.low):
            for w, c in zip(layer, low):
                if c is not None:
                    c.copy_(w)
        for b in self.blocks:
            b.refresh()

    def _read(self, l):
        return [w if c is None else c for w, c in zip(self.W[l], self.low[l])]

    def parameters(self):
        """(weights, bf16 copies or None) in the order of the gradients of a step."""
        w, c = [], []
        for layer, low in zip(self.W, self.low):
            w += [x for x in layer if x is not None]
            c += [y for x, y in zip(layer, low) if x is not None]
        for b in self.blocks:
            w += b.parameters()
            c += [None] * len(b.NAMES)
        return w, c

    def forward(self, X0, ratio, seed, epoch):
        self.inputs, stream, total = [X0], None, 0
        for l in range(self.L):
            Ws, Wn, b = self._read(l)
            _, _, hb = vb.varco_layer_fwd(self.plan, self.inputs[l], Ws, Wn, b, l < self.L - 1, ratio, (seed, epoch, l), self.ws,
                                          F_in=self.widths[l], Y=self.acts[l + 1], Agg=self.aggs[l])
            total += hb
            if l < self.L - 1:
                keep = l > 0 and self.widths[l + 1] == self.widths[l]
                x, stream = self.blocks[l].forward(self.acts[l + 1], stream if keep else None)
                self.inputs.append(x)
        return self.acts[self.L], total

    def step(self, X0, labels, train, ratio, seed, epoch, lr):
        """One step.  Returns (loss as a device scalar, halo bytes of the step); the norm of the averaged gradients before
        clipping is left in self.grad_norm (device scalar)."""
        logits, total = self.forward(X0, ratio, seed, epoch)
        loss, grad = self.loss_and_grad(logits, labels, train)
        layers, blocks, dstream = [None] * self.L, [None] * len(self.blocks), None
        for l in reversed(range(self.L)):
            Ws, Wn, _ = self._read(l)
            dX, dWs, dWn, db, hb = vb.varco_layer_bwd(self.plan, self.inputs[l], self.acts[l + 1], self.aggs[l], Ws, Wn, grad, l < self.L - 1,
                                                      ratio, (seed, epoch, l), self.ws, F_in=self.widths[l], dX=self.grads[l])
            total += hb
            layers[l] = [g for g in (dWs, dWn, db) if g is not None]
            if l > 0:
                grad, blocks[l - 1] = self.blocks[l - 1].backward(dX, dstream)
                keep = l > 1 and self.widths[l] == self.widths[l - 1]
                dstream = grad if keep else None
        weights, copies = self.parameters()
        grads = [g for part in layers + blocks for g in part]
        # the steps of the P workers are averaged: (lr / P) sum_p g_p, clipped by the norm of (1 / P) sum_p g_p
        norm = vb.varco_clip_step(weights, grads, lr / self.P, self.max_norm * self.P, copies=copies, workspace=self.op_ws)
        self.grad_norm = norm / self.P
        for b in self.blocks:
            b.refresh()
        return loss, total

    def status(self):
        """0, or the code of a bounded wait that a kernel of the blocks gave up on (synchronises)."""
        s = [vb.varco_workspace_status(self.op_ws)] + [vb.varco_workspace_status(b.grad_ws) for b in self.blocks]
        return next((x for x in s if x), 0)
