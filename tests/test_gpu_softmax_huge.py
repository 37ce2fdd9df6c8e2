"""Softmax cross-entropy of outputs so large that their rounding errors are whole numbers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")
from gpu_util import force  # noqa: E402
from softmax_util import Reference, inputs  # noqa: E402
from test_gpu_softmax import TILES, run_bwd, run_fwd  # noqa: E402


@pytest.mark.parametrize("tile,splits", [(-1, 0)] + [(t, s) for t in TILES.values() for s in (1, 3)])
@pytest.mark.parametrize("N,I,O", [(100, 256, 300), (300, 700, 1100)])
def test_gradients_of_huge_outputs_are_finite(N, I, O, tile, splits):
    """x and w around 2^12 give outputs around 2^28, off by some 2^5.  An exponential is 1 at most, so that dz, whatever its errors, is no larger than 2 in f16 values with their
    factor: dx is no larger than 2 sum |w|, dw than 2 sum |x|, dbias than 2 N."""
    x, w, b, labels, weight = inputs(N, I, O, 70, "f32", nobody=0.1)
    x, w = 4096 * x, 4096 * I ** 0.5 * w
    ref = Reference(x, w, b, labels)
    with force(tile, splits):
        lse, _, loss = run_fwd(N, I, O, "f32", x, w, b, labels)
        assert np.isfinite(lse).all() and np.isfinite(loss).all()
        for given in (lse, ref.lse.astype(np.float32)):
            got = run_bwd(N, I, O, "f32", x, w, b, labels, given, weight, 1.0, 0.0, None, None)
            for k, most in (("dx", 2.01 * weight[:, None] * np.abs(ref.w).sum(0)), ("dw", 2.01 * (weight[:, None] * np.abs(ref.x)).sum(0)[None, :]), ("db", 2.01 * N)):
                assert np.isfinite(got[k]).all() and (np.abs(got[k]) <= most + 1e-6).all(), (k, np.isfinite(got[k]).mean())
