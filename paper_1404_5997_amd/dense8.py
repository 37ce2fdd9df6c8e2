"""A stack of residual blocks of dense layers in 8 bits, forward, backward and update: how the calls on 8-bit rows are used together.

A block is   h <- h + x;   u = relu(W1 norm(h) + b1);   x <- W2 u + b2   (x: what the block before it gave), and the stack ends in a norm and an
output layer.  Weights live as fp32 masters and as 8-bit rows, which the products read and every update writes anew.

The output layer's units are logistic, or a softmax over the classes.  A softmax is trained without its outputs: the loss and its gradients come from the
normed rows and the layer's weights, both in storage type, so that no buffer has rows of `classes` values however many there are.  (The logits that
`forward` gives come from the weights' 8-bit rows: a served probability differs from the trained one by what 8 bits leave out.)  A bound on the
gradients' norm, where one is given, holds every step back to it.

What a block keeps for its backward pass is h in storage type and, a byte a value, the 8-bit rows that its two products read: they are
operand and checkpoint in one.  u itself is not kept.  Its ReLU mask is read back from the rows: a value that 8 bits took to zero gave
nothing to the product, and gets no gradient.

Buffers and call order only; every arithmetic step runs in the library's kernels.  torch provides device memory.
"""
import torch

from . import (OWT_BF16, OWT_BIAS, OWT_F32, OWT_PASS_BWD_DATA, OWT_PASS_FWD, OWT_RELU, fc_desc, owt_fc_shard_q8_bwd, owt_fc_shard_q8_fwd,
               owt_fc_shard_q8_workspace_bytes, owt_fc_softmax_bwd, owt_fc_softmax_fwd, owt_fc_softmax_workspace_bytes, owt_grad_norm,
               owt_grad_norm_workspace_bytes, owt_logistic_xent, owt_q8_pack, owt_q8_pitch, owt_q8_unpack, owt_rmsnorm_q8_bwd, owt_rmsnorm_q8_fwd,
               owt_rmsnorm_q8_workspace_bytes, owt_sgd_momentum_clipped, owt_sgd_momentum_update, tensor_list)


class Dense8Stack:
    """N rows of `width` values through `blocks` blocks of `hidden` units, then `classes` units: "logistic" ones, or one "softmax" (labels outside
    the classes are then rows that do not count).  max_norm bounds the norm of the gradients of a step (None: no bound)."""

    def __init__(self, N, width, hidden, blocks, classes, dtype="bf16", eps=1e-5, loss="logistic", max_norm=None):
        if loss not in ("logistic", "softmax"):
            raise ValueError("loss is logistic or softmax")
        self.softmax, self.max_norm = loss == "softmax", max_norm
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
        if self.softmax:
            head = self.layers[-1]["desc"]
            scratch = max([scratch] + [owt_fc_softmax_workspace_bytes(head, p) for p in (OWT_PASS_FWD, OWT_PASS_BWD_DATA)])
            self.normed, self.lse = self._new((N, width)), self._new((N,), torch.float32)
        self._carve_parameters()
        self.grad_norm = self._new((1,), torch.float32)
        self._all_grads = tensor_list([self.grads])
        self._lists = [tuple(tensor_list([a[lo:hi]]) for a in (self.params, self.vel, self.grads)) + (None if copy is None else tensor_list([copy]),)
                       for lo, hi, copy in self._ranges]
        scratch = max(scratch, owt_grad_norm_workspace_bytes(self._all_grads))
        self.ws = self._new((max(16, scratch),), torch.uint8)
        self.x = self._new((N, width))          # input, and what a block adds to h
        self.u, self.du = self._new((N, hidden)), self._new((N, hidden))        # one of each for all blocks
        self.dn, self.dh = self._new((N, width)), self._new((N, width))
        self._logits, self.loss = None, self._new((N,), torch.float32)
        self.labels = torch.zeros((N,), device="cuda", dtype=torch.int32)

    @property
    def logits(self):
        """Outputs [N, classes]: made when they are first asked for, which training a softmax never does."""
        if self._logits is None:
            self._logits = self._new((self.N, self.classes))
        return self._logits

    def _new(self, shape, dtype=None):
        return torch.empty(shape, device="cuda", dtype=self.tdt if dtype is None else dtype)

    def _rows(self, cols):
        return self._new((self.N, owt_q8_pitch(cols)), torch.int8)

    def _carve_parameters(self):
        """Weights, biases and gains of the stack in one fp32 array, gradients and momentum in two more: the update is one launch, or two where a part has copies."""
        at, slots = 0, []
        for owner, name, shape in [(e, n, s) for e in self.layers for n, s in (("w", (e["O"], e["I"])), ("b", (e["O"],)))] + \
                                  [(b, "gain", (self.width,)) for b in self.blocks]:
            n = shape[0] * (shape[1] if len(shape) > 1 else 1)
            slots.append((owner, name, shape, at, n))
            at += (n + 7) // 8 * 8              # every view 16-byte aligned
        self.params, self.grads, self.vel = (torch.zeros((at,), device="cuda", dtype=torch.float32) for _ in range(3))
        for owner, name, shape, o, n in slots:
            owner[name], owner["d" + name] = self.params[o:o + n].view(shape), self.grads[o:o + n].view(shape)
        # A softmax reads its layer's weights in storage type: in bf16 every update writes a copy, from those weights on to the array's end (biases and gains).
        head = self.layers[-1]
        self.copies, self._ranges = None, [(0, at, None)]
        if self.softmax and self.tdt == torch.bfloat16:
            o, n = next((o, n) for owner, name, _, o, n in slots if owner is head and name == "w")
            self.copies = torch.zeros((at - o,), device="cuda", dtype=torch.bfloat16)
            self._ranges = [(0, o, None)] * (o > 0) + [(o, at, self.copies)]
            head["stored"] = self.copies[:n].view(head["w"].shape)
        else:
            head["stored"] = head["w"]

    def init(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for e in self.layers:
            e["w"].normal_(0.0, e["I"] ** -0.5, generator=g)
            e["b"].zero_()
        for b in self.blocks:
            b["gain"].fill_(1.0)
        self.pack_weights()

    def pack_weights(self):
        """8-bit rows, and copies in storage type, of the masters as they are."""
        for lo, hi, copy in self._ranges:
            if copy is not None:
                copy.copy_(self.params[lo:hi])
        self._pack_rows()

    def _pack_rows(self):
        for e in self.layers:
            owt_q8_pack(e["O"], e["I"], OWT_F32, e["w"], e["wq"], e["ws"])

    def checkpoint_bytes(self):
        """What the forward pass leaves for the backward pass."""
        return sum(t.numel() * t.element_size() for b in self.blocks for k, t in b.items() if k in ("rstd", "h", "q1", "s1", "q2", "s2"))

    def _shard(self, e, q, s, out):
        owt_fc_shard_q8_fwd(e["desc"], q, s, e["wq"], e["ws"], e["b"], out, self.ws)

    def forward(self, x):
        """Logits [N, classes] of x [N, width] (its own buffer is not written)."""
        self.trunk(x)
        last = self.blocks[-1]
        self._shard(self.layers[-1], last["q1"], last["s1"], self.logits)
        return self.logits

    def trunk(self, x):
        """All blocks and the last norm: what the output layer reads."""
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

    def softmax_loss(self):
        """The losses of the rows that the trunk left, in self.loss."""
        e, b = self.layers[-1], self.blocks[-1]
        owt_q8_unpack(self.N, self.width, self.code, b["q1"], b["s1"], self.normed)
        owt_fc_softmax_fwd(e["desc"], self.normed, e["stored"], e["b"], self.labels, self.lse, None, self.loss, self.ws)

    def _shard_back(self, e, q, s, mask, dy, dx):
        owt_fc_shard_q8_bwd(e["desc"], q, s, e["wq"], e["ws"], mask, dy, 1.0 / self.N, 0.0, dx, e["dw"], e["db"], self.ws)

    def backward(self):
        """Gradients (means over the rows) from the labels; the gradient of the input is left in self.dh."""
        N, code = self.N, self.code
        if self.softmax:
            self.softmax_loss()
        else:
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
            elif self.softmax:
                e, along = self.layers[-1], None
                owt_fc_softmax_bwd(e["desc"], self.normed, e["stored"], e["b"], self.labels, self.lse, None, 1.0 / N, 0.0, self.dn, e["dw"], e["db"], self.ws)
            else:
                self._shard_back(self.layers[-1], b["q1"], b["s1"], None, self.logits, self.dn)
                along = None
            owt_rmsnorm_q8_bwd(N, self.width, code, self.dn, b["h"], b["gain"], b["rstd"], along, 1.0 / N, 0.0, self.dh, b["dgain"], self.ws)

    def update(self, mu, eps, omega):
        if self.max_norm is None:
            for lo, hi, copy in self._ranges:
                owt_sgd_momentum_update(hi - lo, self.params[lo:hi], self.vel[lo:hi], self.grads[lo:hi], mu, eps, omega, -1.0, copy)
        else:
            owt_grad_norm(self._all_grads, OWT_F32, self.grad_norm, self.ws)
            for w, vel, g, copy in self._lists:
                owt_sgd_momentum_clipped(w, vel, g, mu, eps, omega, -1.0, self.grad_norm, self.max_norm, copy)
        self._pack_rows()

    def step(self, x, labels, mu=0.9, eps=0.01, omega=0.0005):
        self.labels.copy_(labels)
        if self.softmax:
            self.trunk(x)
        else:
            self.forward(x)
        self.backward()
        self.update(mu, eps, omega)
