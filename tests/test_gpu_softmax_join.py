"""The join of the workers' shares of a softmax, of very many rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt  # noqa: E402


@pytest.mark.parametrize("N", [1, 256, 257, (1 << 30) + 300])
def test_every_row_is_joined(N):
    """One worker's share is the whole: lse as it was, up to two roundings of a log and a sum; rows without a class are zeros."""
    m = owt()
    lses, targets = (torch.empty((N,), device="cuda") for _ in range(2))
    lses.fill_(3.0)
    targets.fill_(1.0)
    lses[-1], targets[-1] = 5.0, 4.5
    labels = torch.full((N,), 2, device="cuda", dtype=torch.int32)
    if N > 256:
        labels[-2] = -1
    lse, loss = (torch.full((N,), float("nan"), device="cuda") for _ in range(2))
    m.owt_softmax_join(1, N, 7, lses, targets, labels, lse, None, loss)
    torch.cuda.synchronize()
    assert lse[-1].item() == 5.0 and loss[-1].item() == 0.5          # (the log of one is zero)
    if N > 256:
        assert lse[-2].item() == 0.0 and loss[-2].item() == 0.0
        for a, b in ((lse, 3.0), (loss, 2.0)):
            for k in range(0, N - 2, 1 << 27):
                assert (a[k:min(k + (1 << 27), N - 2)] == b).all(), k
