"""Rows without a class have a dx of zeros on every path, also where the weights are not finite."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import force  # noqa: E402
from softmax_util import Reference, inputs  # noqa: E402
from test_gpu_softmax import FEW, TILES, run_bwd  # noqa: E402


@pytest.mark.parametrize("fill", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("N,I,O", [(1, 5, 3), (5, 40, 70), (33, 63, 4100), (64, 130, 257), (70, 130, 257), (300, 64, 600)])
def test_dx_of_padding_beside_weights_that_are_not_finite(N, I, O, fill):
    for dt, tiles in (("f32", [-1, FEW] + list(TILES.values())), ("bf16", [-1] + list(TILES.values()))):
        x, w, b, labels, weight = inputs(N, I, O, 60, dt, nobody=0.3)
        labels[0], labels[-1] = O, -1
        lse = Reference(x, w, b, labels).lse.astype(np.float32)
        w[O // 2, I // 2:] = fill
        w[0, 0] = fill
        for tile in tiles:
            for splits in ((0,) if tile < 0 or tile == FEW else (0, 1, 3)):
                with force(tile, splits):
                    got = run_bwd(N, I, O, dt, x, w, b, labels, lse, weight, 1.0, 0.0, None, None)
                none = (labels < 0) | (labels >= O)
                assert (got["dx"][none] == 0).all(), (dt, tile, splits)
