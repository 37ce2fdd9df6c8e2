"""The operators at the end of a training step whose speed counts, each called as a program calls it, and their plain forms.

A case is one of four kinds:
  loss    softmax cross-entropy of a dense layer's outputs without the outputs: every row's log of the sum of exponentials over the classes,
          its label's output, and their difference, from inputs, weights and bias
  grad    its backward pass from the log of the sum: gradients of inputs, weights and bias.  A row may have a weight, or no class (label -1)
  clip    the norm of the gradients of many tensors together, and those gradients times what brings it down to a bound
  update  the norm, and the momentum / weight-decay update with the bounded gradients, all tensors, with bf16 copies of the weights
"""
import torch

own = False

WIDTHS = (64, 96, 128, 192, 256, 384, 512, 640, 768, 1024, 1152, 1280, 1536, 2048, 2304, 2560, 4096, 4608, 5120, 8192, 9216)
CLASSES = (10, 16, 64, 100, 125, 250, 512, 1000, 1024, 4096, 8192, 10000, 16384, 32000, 32768, 50000, 65536, 100000, 131072)
MU, RATE, DECAY, MAX_NORM = 0.9, 0.01, 0.0005, 1.0


def _loss(name, kind, dtype, N, I, O, masked=False):
    return dict(name=name, kind=kind, dtype=dtype, N=N, I=I, O=O, masked=masked)


def _tensors(name, kind, dtype, blocks, width, hidden, classes):
    return dict(name=name, kind=kind, dtype=dtype, blocks=blocks, width=width, hidden=hidden, classes=classes)


def listed():
    return [
        # the probability of one next token: the weights' bytes are what it costs
        _loss("loss_token_bf16", "loss", "bf16", 1, 4096, 65536),
        # the output layer of the five-layer stack, whole, on one worker's batch
        _loss("loss_classes_f32", "loss", "f32", 128, 4096, 1000),
        # widths and a number of classes that no tile divides, some rows without a class
        _loss("loss_odd_f32", "loss", "f32", 1003, 1025, 32003, masked=True),
        # a training batch's tokens
        _loss("loss_tokens_bf16", "loss", "bf16", 8192, 4096, 32768),
        # a few rows of a large vocabulary: the weights and their gradients are what it costs
        _loss("grad_rows_bf16", "grad", "bf16", 16, 2048, 65536),
        # backward of the five-layer stack's output layer
        _loss("grad_classes_f32", "grad", "f32", 128, 4096, 1000),
        # rows with weights and rows without a class, sizes that no tile divides
        _loss("grad_odd_bf16", "grad", "bf16", 777, 1537, 20011, masked=True),
        # backward of a training batch's tokens
        _loss("grad_tokens_bf16", "grad", "bf16", 4096, 4096, 65536),
        # a small stack of residual blocks: launches and host latency are what it costs
        _tensors("clip_small_f32", "clip", "f32", 3, 96, 250, 10),
        # gradients kept in bf16
        _tensors("clip_blocks_bf16", "clip", "bf16", 6, 2048, 8192, 32768),
        # many small and middling tensors
        _tensors("update_many_f32", "update", "f32", 24, 256, 1021, 1000),
        # a large stack: memory traffic
        _tensors("update_blocks_f32", "update", "f32", 8, 2048, 8192, 1000),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def size(known, lo, hi):        # sizes that layers have, or any
        c = log(lo, hi)
        return c if rng.random() < 0.4 else max(w for w in known if w <= c)

    kind = rng.choice(("loss", "loss", "grad", "grad", "clip", "update"))
    dtype = rng.choice(("f32", "bf16"))
    if kind in ("loss", "grad"):
        most = 4096 * 4096 * 65536 // (1 if dtype == "bf16" else 8)
        while True:
            c = _loss("", kind, dtype, log(1, 8192), size(WIDTHS, 64, 9216), size(CLASSES, 10, 131072), masked=rng.random() < 0.5)
            if c["N"] * c["I"] * c["O"] <= most and c["I"] * c["O"] <= 4096 * 65536 // (1 if dtype == "bf16" else 2):
                break
    else:
        while True:
            c = _tensors("", kind, dtype if kind == "clip" else "f32", rng.randint(1, 32), size(WIDTHS, 64, 2304), size(WIDTHS, 64, 9216), size(CLASSES, 10, 32768))
            if sum(_sizes(c)) <= 8 * 2 * 2048 * 8192:
                break
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)


def _storage(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _sizes(case):
    """Values of each tensor of a stack of residual blocks: two weights, two biases and a gain a block, then gain, weights and bias of the output layer."""
    w, h, c = case["width"], case["hidden"], case["classes"]
    return [h * w, h, w * h, w, w] * case["blocks"] + [w, c * w, c]


def _views(flat, sizes):
    """Tensors one behind the other in one array, each on a 16-byte boundary."""
    got, at = [], 0
    for n in sizes:
        got.append(flat[at:at + n])
        at += (n + 7) // 8 * 8
    return got


def _loss_inputs(case, seed):
    g, t, N, I, O = _gen(seed), _storage(case), case["N"], case["I"], case["O"]
    w = _normal(g, (O, I), 2.0 * I ** -0.5).to(t)
    labels = torch.randint(0, O, (N,), generator=g, device="cuda", dtype=torch.int32)
    # what a trained layer sees: rows that point to their class, some hardly and some clearly
    x = _normal(g, (N, I)).add_(w[labels.long()].float() * (4.0 * torch.rand((N, 1), generator=g, device="cuda")))
    v = dict(x=x.to(t), w=w, b=_normal(g, (O,), 0.1), weight=None)
    if case["masked"]:
        labels = torch.where(torch.rand((N,), generator=g, device="cuda") < 0.1, torch.full_like(labels, -1), labels)
        if case["kind"] == "grad":
            v["weight"] = torch.rand((N,), generator=g, device="cuda", dtype=torch.float32)
    v["labels"] = labels
    if case["kind"] == "grad":
        v["lse"] = torch.where(labels < 0, torch.zeros((), device="cuda"), _plain_lse(v["x"].float() @ w.float().t() + v["b"]))
    return v


def _tensor_inputs(case, seed):
    g, sizes = _gen(seed), _sizes(case)
    n = sum((k + 7) // 8 * 8 for k in sizes)
    inside = torch.zeros((n,), device="cuda")
    for view in _views(inside, sizes):
        view.fill_(1.0)                         # between the tensors there are zeros, which no operator here changes
    v = dict(g=(_normal(g, (n,), 3.0 / n ** 0.5) * inside).to(_storage(case)))      # a norm around three: the bound holds it back
    if case["kind"] == "update":
        v["w"], v["vel"] = _normal(g, (n,), 0.02) * inside, _normal(g, (n,), 1e-4) * inside
    return v


def _inputs(case, seed):
    return (_loss_inputs if case["kind"] in ("loss", "grad") else _tensor_inputs)(case, seed)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    new = lambda shape, d=torch.float32: torch.empty(shape, device="cuda", dtype=d)   # noqa: E731
    if case["kind"] == "clip":
        s["out"] = torch.zeros_like(s["g"])
    elif case["kind"] == "update":
        s["copy"] = torch.zeros_like(s["w"], dtype=torch.bfloat16)
    if own:     # what a program allocates once: results, scratch, lists of tensors
        import paper_1404_5997_amd as owt
        s["code"] = owt.OWT_BF16 if case["dtype"] == "bf16" else owt.OWT_F32
        if case["kind"] in ("loss", "grad"):
            N, I, O = case["N"], case["I"], case["O"]
            s["desc"] = owt.fc_desc(N, I, O, 1, 0, s["code"], owt.OWT_BIAS)
            need = owt.owt_fc_softmax_workspace_bytes(s["desc"], owt.OWT_PASS_FWD if case["kind"] == "loss" else owt.OWT_PASS_BWD_DATA)
            if case["kind"] == "loss":
                s["out"] = dict(lse=new((N,)), target=new((N,)), loss=new((N,)))
            else:
                s["out"] = dict(dx=new((N, I), _storage(case)), dw=new((O, I)), db=new((O,)))
        else:
            sizes = _sizes(case)
            s["lists"] = {k: owt.tensor_list(_views(s[k], sizes)) for k in ("g", "out", "w", "vel", "copy") if k in s}
            need = owt.owt_grad_norm_workspace_bytes(s["lists"]["g"])
            s["norm"] = new((1,))
        s["scratch"] = new((max(16, need),), torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_lse(z):
    top = z.amax(1, keepdim=True)
    return (top + torch.log(torch.exp(z - top).sum(1, keepdim=True))).squeeze(1)


def _plain_loss(s):
    z = s["x"].float() @ s["w"].float().t() + s["b"]
    real = s["labels"] >= 0
    lse = torch.where(real, _plain_lse(z), 0.0)
    target = torch.where(real, z.gather(1, s["labels"].long().clamp_min(0).unsqueeze(1)).squeeze(1), 0.0)
    return dict(lse=lse, target=target, loss=lse - target)


def _plain_grad(s):
    x, w, N = s["x"].float(), s["w"].float(), s["case"]["N"]
    dz = torch.exp(x @ w.t() + s["b"] - s["lse"].unsqueeze(1))
    rows = torch.arange(N, device=dz.device)
    dz[rows, s["labels"].long().clamp_min(0)] -= 1.0
    real = (s["labels"] >= 0).float()
    dz = dz * (real if s["weight"] is None else real * s["weight"]).unsqueeze(1)
    return dict(dx=(dz @ w).to(s["x"].dtype), dw=dz.t() @ x / N, db=dz.sum(0, dtype=torch.float64).float() / N)


def _plain_norm(s):
    """All tensors lie in one array, with zeros between them: a pass over the array is a pass over each."""
    return torch.sqrt(s["g"].double().square().sum()).float()


def _plain_clip(s):
    norm = _plain_norm(s)
    s["out"].copy_(s["g"].float() * torch.clamp(MAX_NORM / norm, max=1.0))
    return dict(norm=norm.reshape(1), out=s["out"])


def _plain_update(s):
    norm = _plain_norm(s)
    factor = torch.clamp(MAX_NORM / norm, max=1.0)
    s["vel"].copy_(MU * s["vel"] - RATE * (factor * s["g"] + DECAY * s["w"]))
    s["w"].add_(s["vel"])
    s["copy"].copy_(s["w"])
    return dict(norm=norm.reshape(1), w=s["w"], vel=s["vel"], copy=s["copy"])


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return dict(loss=_plain_loss, grad=_plain_grad, clip=_plain_clip, update=_plain_update)[kind](s)
    import paper_1404_5997_amd as owt
    if kind == "loss":
        o = s["out"]
        owt.owt_fc_softmax_fwd(s["desc"], s["x"], s["w"], s["b"], s["labels"], o["lse"], o["target"], o["loss"], s["scratch"])
        return o
    if kind == "grad":
        o = s["out"]
        owt.owt_fc_softmax_bwd(s["desc"], s["x"], s["w"], s["b"], s["labels"], s["lse"], s["weight"], 1.0 / c["N"], 0.0, o["dx"], o["dw"], o["db"],
                               s["scratch"])
        return o
    v = s["lists"]
    owt.owt_grad_norm(v["g"], s["code"], s["norm"], s["scratch"])
    if kind == "clip":
        owt.owt_grad_clip(v["g"], v["out"], s["code"], s["norm"], MAX_NORM)
        return dict(norm=s["norm"], out=s["out"])
    owt.owt_sgd_momentum_clipped(v["w"], v["vel"], v["g"], MU, RATE, DECAY, -1.0, s["norm"], MAX_NORM, v["copy"])
    return dict(norm=s["norm"], w=s["w"], vel=s["vel"], copy=s["copy"])


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("loss", "grad"):
        N, I, O = case["N"], case["I"], case["O"]
        if case["kind"] == "loss":
            return dict(bytes=e * I * (N + O) + 4 * (O + 4 * N), flops=2 * N * I * O)
        # the outputs once more, and the two products of their gradients
        return dict(bytes=e * I * (2 * N + O) + 4 * (I * O + 2 * O + 2 * N), flops=6 * N * I * O)
    n = sum(_sizes(case))
    if case["kind"] == "clip":
        return dict(bytes=2 * e * n, flops=3 * n)
    return dict(bytes=(5 * 4 + 2) * n, flops=8 * n)


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits."""
    v, kind, d64 = _inputs(case, seed), case["kind"], torch.float64
    if kind in ("loss", "grad"):
        N, none = case["N"], v["labels"] < 0
        x, w = v["x"].to(d64), v["w"].to(d64)
        z = torch.addmm(v["b"].to(d64), x, w.t().contiguous())
        hot = torch.nn.functional.one_hot(v["labels"].long().clamp_min(0), case["O"]) if N * case["O"] <= 1 << 26 else None
        at = v["labels"].long().clamp_min(0)[:, None]
        if kind == "loss":
            lse, target = torch.logsumexp(z, 1), torch.take_along_dim(z, at, 1)[:, 0]
            lse, target = lse.masked_fill(none, 0.0), target.masked_fill(none, 0.0)
            return dict(lse=lse, target=target, loss=lse - target)
        z = z.sub_(v["lse"].to(d64)[:, None]).exp_()
        if hot is not None:
            z = z - hot
        else:
            z.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=d64))
        factor = (~none).to(d64)
        if v["weight"] is not None:
            factor = factor * v["weight"].to(d64)
        z.mul_(factor[:, None])
        return dict(dx=z @ w, dw=(z.t().contiguous() @ x).div_(N), db=z.sum(0).div_(N))
    g = v["g"].to(d64)
    norm = torch.linalg.vector_norm(g)
    bounded = g * min(1.0, MAX_NORM / norm.item())
    if kind == "clip":
        return dict(norm=norm.reshape(1), out=bounded)
    w, vel = v["w"].to(d64), v["vel"].to(d64)
    # the objective falls along the gradient: the rule, which adds it, gets it negated
    new = MU * vel - RATE * (bounded + DECAY * w)
    return dict(norm=norm.reshape(1), w=w + new, vel=new, copy=w + new)
