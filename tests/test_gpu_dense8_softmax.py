"""The stack of 8-bit dense blocks with a softmax at its end and a bound on its steps: loss, gradients and update against 64 bits on the rows that the stack kept."""
import re

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt  # noqa: E402
from softmax_util import Reference, assert_within, grads  # noqa: E402

U = 2.0 ** -24


def new(N, W, H, B, C, dt, **kw):
    from paper_1404_5997_amd.dense8 import Dense8Stack
    net = Dense8Stack(N, W, H, B, C, dt, **kw)
    net.init(3)
    return net


def batch(N, W, C, seed, net):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((N, W), generator=g, device="cuda").to(net.tdt)
    return x, torch.randint(0, C, (N,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_loss_gradients_and_step(dt):
    owt()
    N, W, H, B, C = 70, 136, 300, 2, 1003
    net = new(N, W, H, B, C, dt, loss="softmax", max_norm=0.05)
    x, labels = batch(N, W, C, 5, net)
    labels[::7] = -1                        # rows that do not count
    net.labels.copy_(labels)
    net.trunk(x)
    net.backward()
    torch.cuda.synchronize()
    e, b = net.layers[-1], net.blocks[-1]
    host = lambda t: t.float().cpu().numpy()   # noqa: E731
    normed = (b["q1"][:, :W].float() * b["s1"][:, None]).to(net.tdt)
    assert torch.equal(net.normed, normed)
    ref = Reference(host(normed), host(e["stored"]), host(e["b"]), labels.cpu().numpy())
    assert_within(host(net.loss), ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")
    want = grads(ref, host(net.lse), None, dt, 1.0 / N, 0.0, None, None)
    for k, t in (("dx", net.dn), ("dw", e["dw"]), ("db", e["db"])):
        if k != "dx" or B == 0:             # (a block's own gradients have since been where dx was)
            assert_within(host(t), *want[k], k)
    # the step
    g, w, v = (t.double().clone() for t in (net.grads, net.params, net.vel))
    net.update(0.9, 0.1, 0.01)
    torch.cuda.synchronize()
    norm = float(g.square().sum().sqrt())
    assert abs(net.grad_norm.item() - norm) <= 1.001 * U * norm and norm > 0.05
    mu, eps, omega, most = (float(np.float32(a)) for a in (0.9, 0.1, 0.01, 0.05))
    step = -g * (most / net.grad_norm.item()) - omega * w
    v2 = mu * v + eps * step
    # the factor, omega w, their sum, its product and the sum with mu v: each rounded once
    off = U * 1.01 * (eps * (1.1 * (step + omega * w).abs() + 1.1 * omega * w.abs() + 2.1 * step.abs()) + v2.abs()) + 2.0 ** -126
    assert ((net.vel.double() - v2).abs() <= off).all()
    assert ((net.params.double() - (w + net.vel.double())).abs() <= U * 1.01 * (w + net.vel.double()).abs()).all()
    assert torch.equal(e["stored"], e["w"].to(net.tdt))
    assert net._logits is None              # no rows of outputs were made


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_dx_of_the_output_layer(dt):
    owt()
    N, W, C = 40, 64, 500
    net = new(N, W, 32, 0, C, dt, loss="softmax")
    x, labels = batch(N, W, C, 6, net)
    net.labels.copy_(labels)
    net.trunk(x)
    net.backward()
    torch.cuda.synchronize()
    e = net.layers[-1]
    host = lambda t: t.float().cpu().numpy()   # noqa: E731
    ref = Reference(host(net.normed), host(e["stored"]), host(e["b"]), labels.cpu().numpy())
    assert_within(host(net.dn), *grads(ref, host(net.lse), None, dt, 1.0 / N, 0.0, None, None)["dx"], "dx")


def test_gradients_that_are_not_finite_move_nothing():
    owt()
    net = new(16, 64, 96, 1, 20, "bf16", loss="softmax", max_norm=1.0)
    x, labels = batch(16, 64, 20, 7, net)
    net.step(x, labels)
    x[3, 5] = float("nan")
    was = net.params.clone()
    net.step(x, labels)
    torch.cuda.synchronize()
    assert not np.isfinite(net.grad_norm.item()) and torch.equal(net.params, was)


def test_two_ways_to_bound_agree_and_no_bound_is_the_plain_update():
    owt()
    N, W, C = 64, 128, 50
    nets = [new(N, W, 256, 1, C, "f32", loss="softmax", max_norm=m) for m in (None, float("inf"))]
    x, labels = batch(N, W, C, 8, nets[0])
    for _ in range(2):
        for net in nets:
            net.step(x, labels, eps=0.05)
    assert torch.equal(nets[0].params, nets[1].params) and torch.equal(nets[0].vel, nets[1].vel)
    with pytest.raises(ValueError):
        new(4, 64, 64, 1, 4, "f32", loss="hinge")


def test_the_example_with_a_softmax(capsys):
    import train_dense8
    train_dense8.main(["--rows", "48", "--width", "128", "--hidden", "256", "--blocks", "1", "--classes", "300", "--steps", "3", "--loss", "softmax", "--max-norm", "0.5"])
    out = capsys.readouterr().out
    assert re.search(r"step 2: loss \d+\.\d+, gradients \d+\.\d+", out), out
    assert re.search(r"single rows: \d+ of 48 right", out), out
    with pytest.raises(SystemExit):
        train_dense8.main(["--max-norm", "0"])


def test_the_convolution_stack_takes_a_bound():
    m = owt()
    from paper_1404_5997_amd.stack import ConvStack
    layers = [dict(K=16, R=3, stride=1, pad=1, pool=True), dict(K=24, R=3, stride=1, pad=1, pool=False)]
    for dt in ("f32", "bf16"):
        net = ConvStack(2, layers, (12, 12, 8), dtype=dt)
        g = torch.Generator(device="cuda").manual_seed(2)
        for a, std in ((net.params, 0.1), (net.grads, 0.5), (net.vel, 0.01)):
            a.normal_(0.0, std, generator=g)
        norm = float(net.grads.double().square().sum().sqrt())
        w, v = net.params.clone(), net.vel.clone()
        copy = torch.zeros_like(w, dtype=torch.bfloat16) if dt == "bf16" else None
        net.update(0.9, 0.01, 0.0005, max_norm=0.25)
        # the same step with the bound in gscale
        m.owt_sgd_momentum_update(net.n_params, w, v, net.grads, 0.9, 0.01, 0.0005, -0.25 / net.grad_norm.item(), copy)
        torch.cuda.synchronize()
        assert abs(net.grad_norm.item() - norm) <= 1.001 * U * norm
        # gscale of the one and the factor of the other are each rounded to fp32 once
        assert ((net.params - w).abs() <= 2.0 ** -23 * w.abs() + 2.0 ** -22 * 0.01 * net.grads.abs()).all()
        if copy is not None:
            assert torch.equal(net.params_bf16, net.params.to(torch.bfloat16))
