"""Bounds so far below the gradients' norm that their ratio is no normal fp32 number: what comes of large gradients is one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt, workspace  # noqa: E402

U = 2.0 ** -24


def tensors(scale):
    g = np.random.default_rng(3)
    return [(scale * g.standard_normal(n)).astype(np.float32) for n in (5, 4096, 4100, 1)]


@pytest.mark.parametrize("scale,most", [(1e36, 1e-3), (1e36, 1.0), (1e30, 1e-12), (1e25, 1e-25), (1e10, 1e-10), (1.0, 0.5), (1e-3, 1e3), (1e30, 1e-40)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_clip_and_update(dt, scale, most):
    m = owt()
    t = torch.bfloat16 if dt == "bf16" else torch.float32
    g = [torch.from_numpy(a).cuda().to(t) for a in tensors(scale)]
    lst, out, norm = m.tensor_list(g), [torch.full_like(a, 7.0) for a in g], torch.empty((1,), device="cuda")
    ws = workspace(m.owt_grad_norm_workspace_bytes(lst))
    code = m.OWT_BF16 if dt == "bf16" else m.OWT_F32
    m.owt_grad_norm(lst, code, norm, ws)
    m.owt_grad_clip(lst, m.tensor_list(out), code, norm, most)
    torch.cuda.synchronize()
    most = float(np.float32(most))
    factor = min(1.0, most / float(norm.item()))
    half = 2.0 ** -8 if dt == "bf16" else U
    for a, o in zip(g, out):
        want = a.double() * factor
        # the factor's rounding, its product's, and storage's; below the normal numbers half a step of theirs (of bf16's, 2^-133, and fp32's)
        off = (2.1 * U + half * 1.01) * want.abs() + (2.0 ** -134 if dt == "bf16" else 2.0 ** -149) + 2.0 ** -149
        assert torch.isfinite(o).all() and ((o.double() - want).abs() <= off).all(), ((o.double() - want).abs() / off).max()
    if dt == "bf16":
        return
    w, vel = ([torch.zeros_like(a) for a in g] for _ in range(2))
    m.owt_sgd_momentum_clipped(m.tensor_list(w), m.tensor_list(vel), lst, 0.0, 1.0, 0.0, -0.5, norm, most)
    torch.cuda.synchronize()
    factor = 0.5 * min(1.0, most / (0.5 * float(norm.item())))
    for a, v in zip(g, vel):
        want = -a.double() * factor
        assert ((v.double() - want).abs() <= 2.1 * U * want.abs() + 2.0 ** -148).all(), ((v.double() - want).abs() / want.abs()).max()
