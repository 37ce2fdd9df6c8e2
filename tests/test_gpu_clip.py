"""The norm of many gradients, gradients and updates that it bounds, against 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt, workspace  # noqa: E402

U = 2.0 ** -24
# one value, nothing, sizes about a chunk of 16 KB and its accesses, more tensors than a launch takes
LISTS = [[], [0], [1], [0, 3, 0], [4095, 4096, 4097], [8191, 8192, 8193, 1], [7] * 200, [4096, 8192, 4095], [4, 3], [5000, 0, 70001] * 60, [1 << 20, 3, (1 << 21) + 5]]


def make(sizes, dtype, seed, scale=1.0):
    """Views of one array, each on a 16-byte boundary, with marked values around them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = 16 + sum((n + 7) // 8 * 8 + 8 for n in sizes)
    flat = torch.full((total,), 7.0, device="cuda", dtype=dtype)
    views, at = [], 8
    for n in sizes:
        views.append(flat[at:at + n])
        views[-1].copy_((torch.randn((n,), generator=g, device="cuda") * scale).to(dtype))
        at += (n + 7) // 8 * 8 + 8
    return flat, views


def outside(flat, views):
    mask = torch.ones_like(flat, dtype=torch.bool)
    for v in views:
        at = (v.data_ptr() - flat.data_ptr()) // flat.element_size()
        mask[at:at + v.numel()] = False
    return flat[mask]


def norm_of(views):
    return float(np.sqrt(sum(float((v.double() ** 2).sum()) for v in views)))


def run_norm(m, views, code):
    lst = m.tensor_list(views)
    need = m.owt_grad_norm_workspace_bytes(lst)
    ws = torch.full((need + 64,), 0x5a, device="cuda", dtype=torch.uint8)
    norm = torch.full((4,), -1.0, device="cuda")
    m.owt_grad_norm(lst, code, norm, ws[:need] if need else None)
    torch.cuda.synchronize()
    assert (ws[need:] == 0x5a).all() and (norm[1:] == -1).all()
    return lst, norm


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("k", range(len(LISTS)))
def test_norm_and_clip(k, dt):
    m = owt()
    code, t = (m.OWT_F32, torch.float32) if dt == "f32" else (m.OWT_BF16, torch.bfloat16)
    flat, views = make(LISTS[k], t, k)
    lst, norm = run_norm(m, views, code)
    want = norm_of(views)
    # the sum is in 64 bits; its root is rounded once
    assert abs(norm[0].item() - want) <= 1.001 * U * want
    before = [v.clone() for v in views]
    half = 2.0 ** -8 if dt == "bf16" else U
    for most in (0.37 * want + 1e-3, 2.0 * want + 1.0, float("inf")):
        out_flat, out = make(LISTS[k], t, 99)
        m.owt_grad_clip(lst, m.tensor_list(out), code, norm, most)
        torch.cuda.synchronize()
        f = min(1.0, most / norm[0].item()) if want else 1.0
        for g, o in zip(before, out):
            # the factor is rounded, then the product, then what is stored
            assert ((o.double() - g.double() * f).abs() <= g.double().abs() * f * (2.5 * U + half) + 2.0 ** -126).all()
        assert (outside(out_flat, out) == 7).all()
    m.owt_grad_clip(lst, lst, code, norm, 0.37 * want + 1e-3)          # in place
    m.owt_grad_clip(lst, lst, code, torch.zeros(4, device="cuda"), 5.0)
    torch.cuda.synchronize()
    f = min(1.0, (0.37 * want + 1e-3) / norm[0].item()) if want else 1.0
    for g, o in zip(before, views):
        assert ((o.double() - g.double() * f).abs() <= g.double().abs() * f * (2.5 * U + half) + 2.0 ** -126).all()
    assert (outside(flat, views) == 7).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_squares_beyond_fp32(dt, scale):
    m = owt()
    _, views = make([1000, 77, 20000], torch.float32 if dt == "f32" else torch.bfloat16, 3, scale)
    _, norm = run_norm(m, views, m.OWT_F32 if dt == "f32" else m.OWT_BF16)
    want = norm_of(views)
    assert abs(norm[0].item() - want) <= 1.001 * U * want


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [(0, 0), (1, 4100), (2, 6)])
def test_a_value_that_is_not_finite(dt, bad, at):
    m = owt()
    code, t = (m.OWT_F32, torch.float32) if dt == "f32" else (m.OWT_BF16, torch.bfloat16)
    flat, views = make([100, 4101, 7], t, 4)
    views[at[0]][at[1]] = bad
    lst, norm = run_norm(m, views, code)
    assert not np.isfinite(norm[0].item())
    _, out = make([100, 4101, 7], t, 5)
    m.owt_grad_clip(lst, m.tensor_list(out), code, norm, 1.0)
    torch.cuda.synchronize()
    assert all((o == 0).all() for o in out)
    if dt == "f32":                         # no step
        (_, w), (_, vel) = make([100, 4101, 7], t, 6), make([100, 4101, 7], t, 7)
        copies = [v.to(torch.bfloat16).clone() for v in out]
        was = [v.clone() for v in w + vel]
        m.owt_sgd_momentum_clipped(m.tensor_list(w), m.tensor_list(vel), lst, 0.9, 0.1, 0.01, -1.0, norm, 1.0, m.tensor_list(copies))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(w + vel, was)) and all((c == 0).all() for c in copies)


@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("k", range(len(LISTS)))
def test_update(k, copy):
    m = owt()
    sizes = LISTS[k]
    (gf, g), (wf, w), (vf, vel), (cf, c) = (make(sizes, t, 10 + j) for j, t in enumerate([torch.float32] * 3 + [torch.bfloat16]))
    lists = [m.tensor_list(v) for v in (w, vel, g, c)]
    mu, eps, omega = 0.9, 0.05, 0.002
    _, norm = run_norm(m, g, m.OWT_F32)
    for gscale, most in ((-1.0, 0.3), (0.25, 1e9), (-0.01, 1e-3), (0.0, 1.0)):
        w0, v0, g0 = ([v.double() for v in a] for a in (w, vel, g))
        m.owt_sgd_momentum_clipped(lists[0], lists[1], lists[2], mu, eps, omega, gscale, norm, most, lists[3] if copy else None)
        torch.cuda.synchronize()
        mu_, eps_, omega_, gscale_, most_ = (float(np.float32(v)) for v in (mu, eps, omega, gscale, most))
        size = abs(gscale_) * norm[0].item()
        f = min(1.0, most_ / size) if size else 1.0
        for w1, v1, c1, a, b, d in zip(w, vel, c, w0, v0, g0):
            step = gscale_ * f * d - omega_ * a
            v2 = mu_ * b + eps_ * step
            # the factor, omega w, their sum, its product and the sum with mu vel: each rounded once
            off = U * (eps_ * (1.1 * (gscale_ * f * d).abs() + 1.1 * omega_ * a.abs() + 2.1 * step.abs()) + v2.abs()) * 1.01 + 2.0 ** -126
            assert ((v1.double() - v2).abs() <= off).all()
            assert ((w1.double() - (a + v1.double())).abs() <= U * (a + v1.double()).abs() * 1.01 + 2.0 ** -126).all()
            if copy:
                assert torch.equal(c1, w1.to(torch.bfloat16))
    assert all((outside(f_, v_) == 7).all() for f_, v_ in ((gf, g), (wf, w), (vf, vel), (cf, c)))


def test_without_a_bound_it_is_the_update_of_one_array():
    m = owt()
    n = 100003
    (_, [g]), (_, [w]), (_, [vel]) = (make([n], torch.float32, 20 + j) for j in range(3))
    w2, v2 = torch.empty((n + 5,), device="cuda")[:n].copy_(w), torch.empty((n + 5,), device="cuda")[:n].copy_(vel)
    _, norm = run_norm(m, [g], m.OWT_F32)
    m.owt_sgd_momentum_clipped(m.tensor_list([w]), m.tensor_list([vel]), m.tensor_list([g]), 0.9, 0.01, 0.0005, -1.0, norm, float("inf"))
    m.owt_sgd_momentum_update(n, w2, v2, g, 0.9, 0.01, 0.0005, -1.0)
    torch.cuda.synchronize()
    assert torch.equal(w, w2) and torch.equal(vel, v2)


def test_captured_and_replayed_and_on_a_stream():
    m = owt()
    sizes = [5000, 33, 90000] * 40
    (_, g), (_, w), (_, vel) = (make(sizes, torch.float32, 30 + j) for j in range(3))
    lists = [m.tensor_list(v) for v in (w, vel, g)]
    ws, norm = workspace(m.owt_grad_norm_workspace_bytes(lists[2])), torch.zeros(1, device="cuda")
    eager = [[v.clone() for v in a] for a in (w, vel)]
    elists = [m.tensor_list(a) for a in eager]

    def step(lw, lv, stream=None):
        m.owt_grad_norm(lists[2], m.OWT_F32, norm, ws, stream)
        m.owt_sgd_momentum_clipped(lw, lv, lists[2], 0.9, 0.01, 0.0005, -1.0, norm, 1.0, None, stream)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(lists[0], lists[1])
    for k in range(3):
        for j, v in enumerate(g):
            v.fill_(0.01 * (k + 1) * (j % 7 - 3))
        graph.replay()
        torch.cuda.synchronize()
        step(*elists, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(w + vel, eager[0] + eager[1])), k
