"""dx of softmax cross-entropy in bf16 keeps 16 bits of dz whatever the layer's size: beside its terms' and sums' errors only the result is rounded.

A row's dz add up to zero, so what all classes' weights have in common cancels in dx, and what dz lost does not.  The weights here have 1 or -1 in common and
differ by some 2^-5."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import force  # noqa: E402
from softmax_util import U, Reference, assert_within  # noqa: E402
from test_gpu_softmax import TILES, run_bwd  # noqa: E402


def cancelling(N, I, O, few_in, few_out, seed):
    """Rows with `few_in` values, classes all but `few_out` of which are taken out: what is zero adds no rounding to a sum however long it is."""
    g = np.random.default_rng(seed)
    common = g.choice([-1.0, 1.0], I)
    w = (common * (1.0 + 2.0 ** -7 * g.integers(0, 8, (O, I)))).astype(np.float32)          # (exact in bf16)
    x = np.zeros((N, I), np.float32)
    x[:, g.permutation(I)[:few_in]] = torch.from_numpy(0.5 * g.standard_normal((N, min(few_in, I)))).bfloat16().float().numpy()
    live = g.permutation(O)[:few_out]
    b = np.full(O, -np.inf, np.float32)
    b[live] = g.standard_normal(len(live))
    labels = g.choice(live, N).astype(np.int32)
    labels[::7] = -1
    return x, w, b, labels, (0.5 + g.random(N)).astype(np.float32)


def bounds(ref, lse, weight, few_in, few_out):
    """dx and how far it may be off: an output's sum starts at bias - lse / 2, each of its terms, cut or rounded, costs 2 U of all that is added up; its exponential is good to 2^-17 of
    itself; two bf16 values are off by 2^-16 of dz; a sum costs 2 U a term that is not zero, and half a step of bf16 is 2^-8."""
    with np.errstate(all="ignore"):
        p = np.where(np.isneginf(ref.z), 0.0, np.exp(ref.z - lse.astype(np.float64)[:, None]))
    d = p.copy()
    d[np.arange(len(d))[ref.mine], ref.at[ref.mine]] -= 1.0
    f = np.where(ref.real, weight.astype(np.float64), 0.0)[:, None]
    size = np.abs(ref.x) @ np.abs(ref.w).T + np.where(np.isfinite(ref.b), np.abs(ref.b), 0.0) + np.abs(lse)[:, None]
    off = 2.0 ** -125 + p * np.expm1(2 * U * (few_in + 3) * size + 2.0 ** -17) + 4 * U * np.abs(d)
    dx = (d * f) @ ref.w
    before = (off * f + np.abs(d * f) * (2.0 ** -16 + 2 * U * (few_out + 2))) @ np.abs(ref.w)
    return dx, before + 2.0 ** -8 * (np.abs(dx) + before)


def check(N, I, O, few_in=16, few_out=40):
    x, w, b, labels, weight = cancelling(N, I, O, few_in, few_out, N + I + O)
    ref = Reference(x, w, b, labels)
    lse = ref.lse.astype(np.float32)
    got = run_bwd(N, I, O, "bf16", x, w, b, labels, lse, weight, 1.0 / N, 0.0, None, None)["dx"]
    assert_within(got, *bounds(ref, lse, weight, few_in, few_out), "dx")
    assert (got[~ref.real] == 0).all()


# small layers (up to 2^28 products and 2^24 weights), and beyond: whole steps and broken ones, few rows and many
@pytest.mark.parametrize("N,I,O", [(100, 64, 100), (2048, 1024, 130), (1000, 2100, 130), (300, 65, 14000), (65, 1030, 4100), (64, 4096, 4100), (16, 4100, 4104), (1100, 512, 600)])
def test_as_planned(N, I, O):
    check(N, I, O)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("N,I,O", [(1100, 512, 600), (300, 130, 7000), (16, 4096, 4100)])
def test_tiles_and_splits(N, I, O, tile, splits):
    with force(TILES[tile], splits):
        check(N, I, O)


def test_in_pieces():
    """Parts of dx are added up in fp32 over pieces of classes."""
    check(16400, 8, 2100, few_in=8)
