"""Softmax cross-entropy whose classes are taken in pieces."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")
from softmax_util import Reference, assert_within, grads, inputs  # noqa: E402
from test_gpu_softmax import run_bwd, run_fwd  # noqa: E402


@pytest.mark.parametrize("N,I,O", [(100, 6400, 8000), (512, 4096, 8000)])
def test_a_short_last_piece_behind_a_long_one(N, I, O):
    """fp32 weights of 4096 classes are laid out four rows a work-group, the 3904 of the last piece one by one: as many words of scratch for their exponents."""
    x, w, b, labels, weight = inputs(N, I, O, 50, "f32")
    ref = Reference(x, w, b, labels)
    lse = ref.lse.astype(np.float32)
    first = None
    for _ in range(3):
        got = run_bwd(N, I, O, "f32", x, w, b, labels, lse, weight, 1.0 / N, 0.0, None, None)
        if first is None:
            for k, (want, off) in grads(ref, lse, weight, "f32", 1.0 / N, 0.0, None, None).items():
                assert_within(got[k], want, off, k)
        else:
            assert all(np.array_equal(first[k], got[k]) for k in got)
        first = got


@pytest.mark.parametrize("dt,N,I,O,piece", [("f32", 65, 8192, 9000, 4608), ("bf16", 65, 8193, 17000, 8704)])
def test_forward_in_pieces(dt, N, I, O, piece):
    """More than 256 MB of weights that are laid out; labels on both sides of where pieces meet, and at both ends."""
    x, w, b, labels, _ = inputs(N, I, O, 51, dt)
    labels[:6] = [piece - 1, piece, 0, O - 1, -1, piece + 1]
    ref = Reference(x, w, b, labels)
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    assert_within(target, ref.target, ref.z_off().max(1), "target")
    assert_within(loss, ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")
