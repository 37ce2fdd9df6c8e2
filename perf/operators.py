"""The operators of a dense layer in 8 bits whose speed counts, each called as a program calls it, and their plain forms.

Rows of 8-bit values stand for real ones: value = q * scale, one scale a row (a token of activations, a channel of weights).
A row of `cols` values takes the next multiple of 128 bytes, zeros behind its values.  A case is one of five kinds:
  norm      h = x + residual, RMS norm of h with a gain, the result in 8 bits with a scale for each row; read back to storage type
  norm_bwd  the norm's backward pass: the gradient of h (with what arrives along the residual path) and that of the gain
  fc        a fully-connected shard's forward pass on 8-bit rows and 8-bit weights, bias + ReLU
  pack      activations put by in 8 bits, and read back
  fc_bwd    a shard's backward pass from its 8-bit checkpoint: ReLU mask, gradients of input, weights and bias
"""
import torch

own = False

ALIGN = 128             # bytes that a row of 8-bit values is rounded up to
EPS = 1e-5
WIDTHS = (16, 32, 64, 96, 128, 192, 256, 384, 512, 640, 768, 1024, 1152, 1280, 1536, 2048, 2304, 2560, 4096, 4608, 5120, 8192, 9216)


def _rows(name, kind, dtype, rows, cols, residual=False):
    return dict(name=name, kind=kind, dtype=dtype, rows=rows, cols=cols, residual=residual)


def _fc(name, kind, dtype, N, I, O, relu=True):
    return dict(name=name, kind=kind, dtype=dtype, N=N, I=I, O=O, relu=relu)


def listed():
    return [
        # one token of a served model: launches and host latency are what it costs
        _rows("norm_token_bf16", "norm", "bf16", 1, 4096, residual=True),
        # rows of an odd number of values: nothing behind the first row is aligned
        _rows("norm_odd_f32", "norm", "f32", 1001, 2049),
        # a training batch's tokens
        _rows("norm_tokens_bf16", "norm", "bf16", 8192, 4096, residual=True),
        # backward on an odd batch of the convolution stack's features (6 x 6 x 256) and on a training batch's tokens
        _rows("norm_bwd_features_f32", "norm_bwd", "f32", 515, 9216, residual=True),
        _rows("norm_bwd_tokens_bf16", "norm_bwd", "bf16", 8192, 4096, residual=True),
        # one token through a whole layer: the weights' bytes are what it costs
        _fc("fc_token_bf16", "fc", "bf16", 1, 4096, 4096, relu=False),
        # the first dense shard of the five-layer stack, one worker's batch
        _fc("fc_shard_f32", "fc", "f32", 128, 9216, 512),
        # a training batch's tokens through a wide layer
        _fc("fc_tokens_bf16", "fc", "bf16", 8192, 4096, 8192),
        # the checkpoint of the last shard's 125 columns for the batches of eight workers, and of a training batch's tokens
        _rows("pack_shard_f32", "pack", "f32", 1024, 125),
        _rows("pack_tokens_bf16", "pack", "bf16", 16384, 4096),
        # backward of the first dense shard, and of a square layer on a training batch's tokens
        _fc("fc_bwd_shard_f32", "fc_bwd", "f32", 128, 9216, 512),
        _fc("fc_bwd_tokens_bf16", "fc_bwd", "bf16", 8192, 4096, 4096, relu=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def width(lo, hi):      # widths that layers have, or any
        c = log(lo, hi)
        return c if rng.random() < 0.4 else max(w for w in WIDTHS if w <= c)

    kind = rng.choice(("norm", "norm_bwd", "fc", "fc", "pack", "fc_bwd", "fc_bwd"))
    dtype = rng.choice(("f32", "bf16"))
    if kind in ("fc", "fc_bwd"):
        most = 8192 * 4096 * (8192 if kind == "fc" else 4096 if dtype == "bf16" else 2048)
        while True:
            c = _fc("", kind, dtype, log(1, 8192), width(64, 9216), width(16, 8192), relu=rng.random() < 0.5)
            if c["N"] * c["I"] * c["O"] <= most:
                break
    else:
        most = (8192 * 4096 if kind != "pack" else 16384 * 4096) // (2 if dtype == "f32" else 1)
        while True:
            c = _rows("", kind, dtype, log(1, 16384), width(64, 9216), residual=kind != "pack" and rng.random() < 0.7)
            if c["rows"] * c["cols"] <= most:
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


def _pitch(cols):
    return (cols + ALIGN - 1) // ALIGN * ALIGN


def _quantised(t):
    """8-bit rows and scales of fp32 rows, as a program has them in hand: [rows][pitch] bytes, zeros behind the values."""
    amax = t.abs().amax(1, keepdim=True)
    q = torch.zeros((t.shape[0], _pitch(t.shape[1])), device=t.device, dtype=torch.int8)
    q[:, :t.shape[1]] = (t * (127.0 / amax.clamp_min(1e-20))).round().to(torch.int8)
    return q, (amax / 127.0).squeeze(1)


def _inputs(case, seed):
    g, t, kind = _gen(seed), _storage(case), case["kind"]
    if kind in ("fc", "fc_bwd"):
        N, I, O = case["N"], case["I"], case["O"]
        # tokens of different sizes; weights as a layer of this width is initialised
        xq, xs = _quantised(_normal(g, (N, I)) * (0.5 + torch.rand((N, 1), generator=g, device="cuda")))
        wq, ws = _quantised(_normal(g, (O, I), I ** -0.5))
        v = dict(xq=xq, xs=xs, wq=wq, ws=ws)
        if kind == "fc":
            v["b"] = _normal(g, (O,), 0.01)
        else:
            v["dy"] = _normal(g, (N, O), 0.1).to(t)
            v["y"] = _normal(g, (N, O)).relu_().to(t) if case["relu"] else None
        return v
    rows, cols = case["rows"], case["cols"]
    x = _normal(g, (rows, cols)).to(t)
    if kind == "pack":
        return dict(x=x.relu_())                                    # activations behind a ReLU
    v = dict(x=x, gain=_normal(g, (cols,), 0.1).add_(1.0), res=_normal(g, (rows, cols), 2.0).to(t) if case["residual"] else None)
    if kind == "norm_bwd":                                           # x is the sum that was normed
        v["rstd"] = (x.float().square().mean(1) + EPS).rsqrt()
        v["dy"] = _normal(g, (rows, cols)).to(t)
    return v


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if own:     # what a program allocates once: results and scratch
        import paper_1404_5997_amd as owt
        t, kind = _storage(case), case["kind"]
        new = lambda shape, d=t: torch.empty(shape, device="cuda", dtype=d)   # noqa: E731
        f32 = torch.float32
        s["code"] = owt.OWT_BF16 if case["dtype"] == "bf16" else owt.OWT_F32
        need = 0
        if kind in ("fc", "fc_bwd"):
            N, I, O = case["N"], case["I"], case["O"]
            s["desc"] = owt.fc_desc(N, I, O, 1, 0, s["code"], owt.OWT_BIAS | (owt.OWT_RELU if case["relu"] else 0))
            need = owt.owt_fc_shard_q8_workspace_bytes(s["desc"], owt.OWT_PASS_FWD if kind == "fc" else owt.OWT_PASS_BWD_DATA)
            if kind == "fc":
                s["out"] = new((N, O))
            else:
                s["dx"], s["dw"], s["db"] = new((N, I)), new((O, I), f32), new((O,), f32)
        else:
            rows, cols = case["rows"], case["cols"]
            if kind == "norm_bwd":
                s["dx"], s["dgain"] = new((rows, cols)), new((cols,), f32)
                need = owt.owt_rmsnorm_q8_workspace_bytes(rows, cols)
            else:
                s["q"], s["scale"], s["values"] = new((rows, owt.owt_q8_pitch(cols)), torch.int8), new((rows,), f32), new((rows, cols))
                if kind == "norm":
                    s["h"], s["rstd"] = new((rows, cols)) if case["residual"] else None, new((rows,), f32)
        s["scratch"] = new((max(16, need),), torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_q8(t):
    """Whole numbers to 127 and each row's largest magnitude over 127.  Rows of magnitudes near the smallest of fp32 are scaled
    by 2^64 on the way; a row whose largest magnitude is not finite is not finite anywhere (0 times its scale)."""
    amax = t.abs().amax(1, keepdim=True)
    up = torch.where(amax < 2.0 ** -64, 2.0 ** 64, 1.0)
    fine = (amax > 0) & (amax < float("inf"))
    q = torch.where(fine, torch.round(t * up * (127.0 * torch.reciprocal(amax * up))), torch.zeros_like(t))
    return q, amax / 127.0


def _plain_norm(s):
    t = s["x"].dtype
    h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    q, scale = _plain_q8(h * s["gain"])
    scale = scale * rstd
    return dict(h=None if s["res"] is None else h.to(t), rstd=rstd.squeeze(1), scale=scale.squeeze(1), values=(q * scale).to(t))


def _plain_norm_bwd(s):
    h, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"].unsqueeze(1)
    xn, g = h * rstd, dy * s["gain"]
    dx = rstd * (g - xn * (g * xn).mean(1, keepdim=True))
    if s["res"] is not None:
        dx = dx + s["res"].float()
    return dict(dx=dx.to(s["x"].dtype), dgain=(dy * xn).sum(0))


def _plain_fc(s):
    c = s["case"]
    acc = s["xq"][:, :c["I"]].float() @ s["wq"][:, :c["I"]].float().t()
    y = acc * s["xs"].unsqueeze(1) * s["ws"] + s["b"]
    return (y.clamp_min(0.0) if c["relu"] else y).to(_storage(c))


def _plain_fc_bwd(s):
    c = s["case"]
    dz = s["dy"].float()
    if s["y"] is not None:
        dz = dz * (s["y"] > 0)
    dx = (dz * s["ws"]) @ s["wq"][:, :c["I"]].float()
    dw = (dz * s["xs"].unsqueeze(1)).t() @ s["xq"][:, :c["I"]].float() / c["N"]
    return dict(dx=dx.to(_storage(c)), dw=dw, db=dz.sum(0) / c["N"])


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        if kind == "norm":
            return _plain_norm(s)
        if kind == "norm_bwd":
            return _plain_norm_bwd(s)
        if kind == "fc":
            return _plain_fc(s)
        if kind == "fc_bwd":
            return _plain_fc_bwd(s)
        q, scale = _plain_q8(s["x"].float())
        return dict(scale=scale.squeeze(1), values=(q * scale).to(s["x"].dtype))
    import paper_1404_5997_amd as owt
    if kind == "norm":
        owt.owt_rmsnorm_q8_fwd(c["rows"], c["cols"], s["code"], s["x"], s["res"], s["gain"], EPS, s["h"], s["q"], s["scale"], s["rstd"])
        owt.owt_q8_unpack(c["rows"], c["cols"], s["code"], s["q"], s["scale"], s["values"])
        return dict(h=s["h"], rstd=s["rstd"], scale=s["scale"], values=s["values"])
    if kind == "norm_bwd":
        owt.owt_rmsnorm_q8_bwd(c["rows"], c["cols"], s["code"], s["dy"], s["x"], s["gain"], s["rstd"], s["res"], 1.0, 0.0, s["dx"],
                               s["dgain"], s["scratch"])
        return dict(dx=s["dx"], dgain=s["dgain"])
    if kind == "fc":
        owt.owt_fc_shard_q8_fwd(s["desc"], s["xq"], s["xs"], s["wq"], s["ws"], s["b"], s["out"], s["scratch"])
        return s["out"]
    if kind == "fc_bwd":
        owt.owt_fc_shard_q8_bwd(s["desc"], s["xq"], s["xs"], s["wq"], s["ws"], s["y"], s["dy"], 1.0 / c["N"], 0.0, s["dx"], s["dw"],
                                s["db"], s["scratch"])
        return dict(dx=s["dx"], dw=s["dw"], db=s["db"])
    owt.owt_q8_pack(c["rows"], c["cols"], s["code"], s["x"], s["q"], s["scale"])
    owt.owt_q8_unpack(c["rows"], c["cols"], s["code"], s["q"], s["scale"], s["values"])
    return dict(scale=s["scale"], values=s["values"])


def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind in ("fc", "fc_bwd"):
        N, I, O = case["N"], case["I"], case["O"]
        if kind == "fc":
            return dict(bytes=N * I + O * I + N * O * e + 4 * (N + 2 * O), flops=2 * N * I * O)
        return dict(bytes=N * I + O * I + N * O * e * (2 if case["relu"] else 1) + N * I * e + 4 * (O * I + N + 2 * O), flops=4 * N * I * O)
    rows, n = case["rows"], case["rows"] * case["cols"]
    if kind == "norm":      # x, (residual, h), 8-bit values, values read back
        return dict(bytes=n * (e * (4 if case["residual"] else 2) + 1) + 8 * rows + 4 * case["cols"], flops=8 * n)
    if kind == "norm_bwd":
        return dict(bytes=n * e * (4 if case["residual"] else 3) + 4 * rows + 8 * case["cols"], flops=12 * n)
    return dict(bytes=n * (2 * e + 1) + 4 * rows, flops=4 * n)


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """What run() returns, from the definitions in 64 bits."""
    v, kind = _inputs(case, seed), case["kind"]
    d = {k: x.to(torch.float64) for k, x in v.items() if x is not None}

    def eight_bits(t, factor):
        """Every value to the nearest of 255 evenly spaced ones up to its row's largest magnitude, times the row's factor."""
        largest = torch.linalg.vector_norm(t, float("inf"), dim=1)
        unit = largest / 127
        whole = torch.where(largest[:, None] > 0, torch.round(t / torch.where(unit > 0, unit, 1.0)[:, None]), 0.0)
        return unit * factor, whole * (unit * factor)[:, None]

    if kind == "pack":
        scale, values = eight_bits(d["x"], 1.0)
        return dict(scale=scale, values=values)
    if kind == "norm":
        h = d["x"] + d["res"] if "res" in d else d["x"]
        rstd = (torch.einsum("rc,rc->r", h, h) / h.shape[1] + EPS) ** -0.5
        scale, values = eight_bits(h * d["gain"][None, :], rstd)
        return dict(h=h if "res" in d else None, rstd=rstd, scale=scale, values=values)
    if kind == "norm_bwd":
        # d/dh of g x rstd(h): rstd dy g - h rstd^3 <dy g, h> / cols
        along = torch.einsum("rc,rc,c->r", d["dy"], d["x"], d["gain"]) / case["cols"]
        dx = d["rstd"][:, None] * d["dy"] * d["gain"] - d["x"] * (d["rstd"] ** 3 * along)[:, None]
        return dict(dx=dx + d["res"] if "res" in d else dx, dgain=torch.einsum("rc,rc,r->c", d["dy"], d["x"], d["rstd"]))
    x = d["xq"][:, :case["I"]] * d["xs"][:, None]
    w = d["wq"][:, :case["I"]] * d["ws"][:, None]
    if kind == "fc":
        y = torch.addmm(d["b"], x, w.t().contiguous())
        return torch.relu(y) if case["relu"] else y
    dz = torch.where(d["y"] > 0, d["dy"], 0.0) if "y" in d else d["dy"]
    return dict(dx=dz @ w, dw=(dz.t().contiguous() @ x) / case["N"], db=dz.sum(0) / case["N"])
