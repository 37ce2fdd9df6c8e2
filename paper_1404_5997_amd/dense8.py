"""A stack of residual blocks of dense layers in 8 bits, forward, backward and update: how the calls on 8-bit rows are used together.

A block is   h <- h + x;   u = relu(W1 norm(h) + b1);   x <- W2 u + b2   (x: what the block before it gave), and the stack ends in a norm and an
output layer of logistic units.  Weights live as fp32 masters and as 8-bit rows, which the products read and every update writes anew.

What a block keeps for its backward pass is h in storage type and, a byte a value, the 8-bit rows that its two products read: they are
operand and checkpoint in one.  u itself is not kept.  Its ReLU mask is read back from the rows: a value that 8 bits took to zero gave
nothing to the product, and gets no gradient.

Buffers and call order only; every arithmetic step runs in the library's kernels.  torch provides device memory.
"""
import torch

from . import (OWT_BF16, OWT_BIAS, OWT_F32, OWT_PASS_BWD_DATA, OWT_PASS_FWD, OWT_RELU, fc_desc, owt_fc_shard_q8_bwd, owt_fc_shard_q8_fwd,
               owt_fc_shard_q8_workspace_bytes, owt_logistic_xent, owt_q8_pack, owt_q8_pitch, owt_q8_unpack, owt_rmsnorm_q8_bwd,
               owt_rmsnorm_q8_fwd, owt_rmsnorm_q8_workspace_bytes, owt_sgd_momentum_update)


class Dense8Stack:
    """N rows of `width` values through `blocks` blocks of `hidden` units, then `classes` logistic units."""

    def __init__(self, N, width, hidden, blocks, classes, dtype="bf16", eps=1e-5):
        self.N, self.width, self.hidden, self.classes, self.eps = N, width, hidden, classes, eps
        self.code = OWT_BF16 if dtype == "bf16" else OWT_F32
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.layers, self.blocks = [], []
        sizes = [(width, hidden, OWT_BIAS | OWT_RELU), (hidden, width, OWT_BIAS)] * blocks + [(width, classes, OWT_BIAS)]
        scratch = owt_rmsnorm_q8_workspace_bytes(N, width)
        for I, O, flags in sizes:
            e = dict(desc=fc_desc(N, I, O, 1, 0, self.code, flags), I=I, O=O, wq=self._new((O, owt_q8_pitch(I)), torch.int8), ws=self._new((O,), torch.float32))
            scratch = max([scratch] + [owt_fc_shard_q8_workspace_bytes(e["desc"], p) for p in (OWT_PASS_FWD, OWT_PASS_BWD_DATA)])
            self.layers.append(e)
        for _ in range(blocks + 1):             # the last one is the norm in front of the output layer
            b = dict(rstd=self._new((N,), torch.float32), h=self._new((N, width)), q1=self._rows(width), s1=self._new((N,), torch.float32))
            if len(self.blocks) < blocks:
                b.update(q2=self._rows(hidden), s2=self._new((N,), torch.float32))
            self.blocks.append(b)
        self._carve_parameters()
        self.ws = self._new((max(16, scratch),), torch.uint8)
        self.x = self._new((N, width))          # input, and what a block adds to h
        self.u, self.du = self._new((N, hidden)), self._new((N, hidden))        # one of each for all blocks
        self.dn, self.dh = self._new((N, width)), self._new((N, width))
        self.logits, self.loss = self._new((N, classes)), self._new((N,), torch.float32)
        self.labels = torch.zeros((N,), device="cuda", dtype=torch.int32)

    def _new(self, shape, dtype=None):
        return torch.empty(shape, device="cuda", dtype=self.tdt if dtype is None else dtype)

    def _rows(self, cols):
        return self._new((self.N, owt_q8_pitch(cols)), torch.int8)

    def _carve_parameters(self):
        """Weights, biases and gains of the stack in one fp32 array, gradients and momentum in two more: the update is one launch."""
        at, slots = 0, []
        for owner, name, shape in [(e, n, s) for e in self.layers for n, s in (("w", (e["O"], e["I"])), ("b", (e["O"],)))] + \
                                  [(b, "gain", (self.width,)) for b in self.blocks]:
            n = shape[0] * (shape[1] if len(shape) > 1 else 1)
            slots.append((owner, name, shape, at, n))
            at += (n + 7) // 8 * 8              # every view 16-byte aligned
        self.params, self.grads, self.vel = (torch.zeros((at,), device="cuda", dtype=torch.float32) for _ in range(3))
        for owner, name, shape, o, n in slots:
            owner[name], owner["d" + name] = self.params[o:o + n].view(shape), self.grads[o:o + n].view(shape)

    def init(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for e in self.layers:
            e["w"].normal_(0.0, e["I"] ** -0.5, generator=g)
            e["b"].zero_()
        for b in self.blocks:
            b["gain"].fill_(1.0)
        self.pack_weights()

    def pack_weights(self):
        for e in self.layers:
            owt_q8_pack(e["O"], e["I"], OWT_F32, e["w"], e["wq"], e["ws"])

    def checkpoint_bytes(self):
        """What the forward pass leaves for the backward pass."""
        return sum(t.numel() * t.element_size() for b in self.blocks for k, t in b.items() if k in ("rstd", "h", "q1", "s1", "q2", "s2"))

    def _shard(self, e, q, s, out):
        owt_fc_shard_q8_fwd(e["desc"], q, s, e["wq"], e["ws"], e["b"], out, self.ws)

    def forward(self, x):
        """Logits [N, classes] of x [N, width] (its own buffer is not written)."""
        N, last = self.N, None
        for i, b in enumerate(self.blocks):
            if i == 0:
                b["h"].copy_(x)
                owt_rmsnorm_q8_fwd(N, self.width, self.code, b["h"], None, b["gain"], self.eps, None, b["q1"], b["s1"], b["rstd"])
            else:
                owt_rmsnorm_q8_fwd(N, self.width, self.code, self.x, last["h"], b["gain"], self.eps, b["h"], b["q1"], b["s1"], b["rstd"])
            if "q2" in b:
                self._shard(self.layers[2 * i], b["q1"], b["s1"], self.u)
                owt_q8_pack(N, self.hidden, self.code, self.u, b["q2"], b["s2"])
                self._shard(self.layers[2 * i + 1], b["q2"], b["s2"], self.x)
            last = b
        self._shard(self.layers[-1], last["q1"], last["s1"], self.logits)
        return self.logits

    def _shard_back(self, e, q, s, mask, dy, dx):
        owt_fc_shard_q8_bwd(e["desc"], q, s, e["wq"], e["ws"], mask, dy, 1.0 / self.N, 0.0, dx, e["dw"], e["db"], self.ws)

    def backward(self):
        """Gradients (means over the rows) from the labels; the gradient of the input is left in self.dh."""
        N, code = self.N, self.code
        owt_logistic_xent(N, self.classes, 0, code, self.logits, self.labels, 1.0, self.loss, self.logits)
        for i in range(len(self.blocks) - 1, -1, -1):
            b = self.blocks[i]
            if "q2" in b:
                # what a block gives is added to h: its gradient is that of the h behind it
                w1, w2 = self.layers[2 * i], self.layers[2 * i + 1]
                self._shard_back(w2, b["q2"], b["s2"], None, self.dh, self.du)
                owt_q8_unpack(N, self.hidden, code, b["q2"], b["s2"], self.u)
                self._shard_back(w1, b["q1"], b["s1"], self.u, self.du, self.dn)
                along = self.dh
            else:
                self._shard_back(self.layers[-1], b["q1"], b["s1"], None, self.logits, self.dn)
                along = None
            owt_rmsnorm_q8_bwd(N, self.width, code, self.dn, b["h"], b["gain"], b["rstd"], along, 1.0 / N, 0.0, self.dh, b["dgain"], self.ws)

    def update(self, mu, eps, omega):
        owt_sgd_momentum_update(self.params.numel(), self.params, self.vel, self.grads, mu, eps, omega, -1.0)
        self.pack_weights()

    def step(self, x, labels, mu=0.9, eps=0.01, omega=0.0005):
        self.labels.copy_(labels)
        self.forward(x)
        self.backward()
        self.update(mu, eps, omega)
