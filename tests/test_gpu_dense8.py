"""The stack of 8-bit dense blocks: every stage against 64 bits on the rows that the stack itself kept, and training."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt, to_host  # noqa: E402


def values(q, s, cols):
    return q[:, :cols].double() * s.double()[:, None]


def close(got, want, tol):
    """Against the largest value of a tensor, as the framework's parity tests have it."""
    e = ((got.double() - want).abs().max() / want.abs().max()).item()
    assert e <= tol, e


# storage type's rounding (2^-8, 2^-24) of each result, and of what it was summed from
TOL = {"f32": 1e-5, "bf16": 1e-2}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_stages_against_64_bits(dt):
    owt()
    from paper_1404_5997_amd.dense8 import Dense8Stack
    N, W, H, B, C = 70, 136, 300, 2, 25
    net = Dense8Stack(N, W, H, B, C, dt)
    net.init(3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((N, W), generator=g, device="cuda").to(net.tdt)
    labels = torch.randint(0, C, (N,), generator=g, device="cuda", dtype=torch.int32)
    net.labels.copy_(labels)
    logits = net.forward(x).double().clone()
    tol = TOL[dt]
    h = x.double()
    for i, b in enumerate(net.blocks):
        close(b["h"], h, tol)
        n = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * b["gain"].double()
        v = values(b["q1"], b["s1"], W)
        assert (v - n).abs().max() <= 0.51 * b["s1"].max() + 4 * tol * n.abs().max()        # half a unit of 8 bits, and h's rounding
        if "q2" not in b:
            break
        w1, w2 = net.layers[2 * i], net.layers[2 * i + 1]
        u = torch.relu(v @ values(w1["wq"], w1["ws"], W).t() + w1["b"].double())
        uq = values(b["q2"], b["s2"], H)
        assert (uq - u).abs().max() <= 0.51 * b["s2"].max() + tol * u.abs().max()
        h = b["h"].double() + uq @ values(w2["wq"], w2["ws"], H).t() + w2["b"].double()
    out = net.layers[-1]
    close(logits, v @ values(out["wq"], out["ws"], W).t() + out["b"].double(), tol)

    net.backward()
    dz = torch.sigmoid(logits)
    dz[torch.arange(N), labels.long()] -= 1
    b = net.blocks[-1]
    close(out["dw"], dz.t() @ values(b["q1"], b["s1"], W) / N, 2 * tol)
    close(out["db"], dz.sum(0) / N, 2 * tol)
    dn, along = dz @ values(out["wq"], out["ws"], W), 0.0
    for i in range(B, -1, -1):
        b = net.blocks[i]
        hh, r, gain = b["h"].double(), b["rstd"].double()[:, None], b["gain"].double()
        xn = hh * r
        close(b["dgain"], (dn * xn).sum(0) / N, 4 * tol)
        dh = r * (gain * dn - xn * (gain * dn * xn).mean(1, keepdim=True)) + along
        if i == 0:
            break
        w1, w2, p = net.layers[2 * i - 2], net.layers[2 * i - 1], net.blocks[i - 1]
        uq = values(p["q2"], p["s2"], H)
        close(w2["dw"], dh.t() @ uq / N, 4 * tol)
        du = (dh @ values(w2["wq"], w2["ws"], H)) * (uq > 0)
        close(w1["dw"], du.t() @ values(p["q1"], p["s1"], W) / N, 4 * tol)
        close(w1["db"], du.sum(0) / N, 4 * tol)
        dn, along = du @ values(w1["wq"], w1["ws"], W), dh
    close(net.dh, dh, 4 * tol)


def test_training_lowers_the_loss_and_single_rows_agree():
    owt()
    from paper_1404_5997_amd.dense8 import Dense8Stack
    N, W, H, B, C = 256, 128, 512, 2, 10
    net, one = Dense8Stack(N, W, H, B, C, "bf16"), Dense8Stack(1, W, H, B, C, "bf16")
    net.init(0)
    g = torch.Generator(device="cuda").manual_seed(1)
    centres = torch.randn((C, W), generator=g, device="cuda")
    losses = []
    for _ in range(30):
        labels = torch.randint(0, C, (N,), generator=g, device="cuda", dtype=torch.int32)
        x = (centres[labels.long()] + 0.5 * torch.randn((N, W), generator=g, device="cuda")).to(torch.bfloat16)
        net.step(x, labels, eps=0.02)
        losses.append(net.loss.mean().item())
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], losses
    one.params.copy_(net.params)
    one.pack_weights()
    whole = to_host(net.forward(x))
    for i in (0, 17, N - 1):       # whole sums are exact and a row's rounding is its own: the same bits in any batch
        np.testing.assert_array_equal(to_host(one.forward(x[i:i + 1]))[0], whole[i])
    # h in 2 bytes, norm rows and hidden rows in 1, three figures a row
    assert net.checkpoint_bytes() <= N * ((B + 1) * (3 * W + 8) + B * (H + 4))
