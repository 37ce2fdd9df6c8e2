"""dx of the dense shard in 8 bits keeps as many bits of dz * wscale in bf16 as in fp32, whichever kernel serves it: only the result is rounded.

Tolerances are the bounds that the header states, element by element: a value of dz * wscale is off by 2^-22 of itself (both forms hold that, the one
of three bf16 parts more) behind an fp32 rounding (U), and 2^-39 of the row's largest; the fp32 sum of K terms in two or three parts takes at most
2 K / 8 + 16 roundings, each with half a unit of what the instruction drops; and the result is rounded once, to 2^-8 of itself in bf16 (U in fp32)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import force, owt  # noqa: E402
from test_gpu_q8 import U, UB, Shard, say, stored  # noqa: E402

# the plan's choice; the products in tiles of 256, 128 and 64; one launch
KERNELS = [-1, 110, 111, 112, 114]


def check_dx(s):
    dz = np.where(s.y > 0, s.dy, 0).astype(np.float64) if s.relu else s.dy.astype(np.float64)
    w = s.values()[1]
    gx, _, _ = s.backward(1.0, 0.0)
    want, terms = dz @ w, np.abs(dz) @ np.abs(w)
    largest = np.abs(dz * s.ws).max(1)[:, None]
    before = (2.0 ** -22 + U + (2 * s.O / 8 + 16) * 2 * U) * terms + 2.0 ** -38 * largest * np.abs(s.wq[:, :s.I]).sum(0) + 1e-37
    tol = before + 1.01 * (UB if s.dt == "bf16" else U) * (np.abs(want) + before)
    assert np.all(np.abs(gx - want) <= tol), (np.max(np.abs(gx - want) / tol), int((np.abs(gx - want) > tol).sum()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("N,I,O", [(70, 129, 33), (300, 257, 190), (65, 640, 500)])
def test_sums_of_random_terms(N, I, O, kernel, dt):
    """Some of them are small beside their terms."""
    say("case dx bits", N, I, O, kernel, dt)
    with force(kernel):
        check_dx(Shard(N, I, O, dt))
        check_dx(Shard(N, I, O, dt, relu=False, bias=False))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kernel", KERNELS)
def test_two_weights_that_almost_cancel(kernel, dt):
    """dx = dz * wq * (a - b) with b within 2^-12 of a: what dz * a and dz * b lost would stand in the result's first bits."""
    say("case dx that cancels", kernel, dt)
    s = Shard(70, 140, 2, dt, relu=False)
    g = np.random.default_rng(9)
    s.wq[1] = s.wq[0]
    a = np.float32(0.01 * np.exp(g.uniform(-1, 1)))
    s.ws = np.array([a, a * np.float32(1 + 2.0 ** -12)], dtype=np.float32)
    s.dy = np.ascontiguousarray(np.repeat(stored(g.standard_normal((70, 1)), dt), 2, axis=1)) * np.array([1, -1], dtype=np.float32)
    with force(kernel):
        check_dx(s)
