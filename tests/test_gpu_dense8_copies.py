"""The softmax layer's weights in storage type beside the masters of a stack of 8-bit dense blocks: copies of what is read, as every step leaves it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt  # noqa: E402
from test_gpu_dense8_softmax import batch, new  # noqa: E402


@pytest.mark.parametrize("blocks", [0, 2])
@pytest.mark.parametrize("max_norm", [None, 0.05, float("inf")])
def test_copies_of_the_output_layer_alone(blocks, max_norm):
    m = owt()
    N, W, H, C = 33, 72, 200, 301
    net = new(N, W, H, blocks, C, "bf16", loss="softmax", max_norm=max_norm)
    # (weights, and behind them biases and gains, each on a multiple of eight values)
    assert net.copies.numel() <= C * W + (C + 7) // 8 * 8 + (blocks + 1) * W
    head = net.layers[-1]
    assert head["stored"].dtype == torch.bfloat16 and head["stored"].shape == head["w"].shape
    x, labels = batch(N, W, C, 9, net)
    for _ in range(3):
        net.labels.copy_(labels)
        net.trunk(x)
        net.backward()
        w, v = net.params.clone(), net.vel.clone()
        net.update(0.9, 0.1, 0.01)
        # the same step of the whole array in one call
        if max_norm is None:
            m.owt_sgd_momentum_update(w.numel(), w, v, net.grads, 0.9, 0.1, 0.01, -1.0)
        else:
            m.owt_sgd_momentum_clipped(m.tensor_list([w]), m.tensor_list([v]), m.tensor_list([net.grads]), 0.9, 0.1, 0.01, -1.0, net.grad_norm, max_norm)
        torch.cuda.synchronize()
        assert torch.equal(net.params, w) and torch.equal(net.vel, v)
        assert torch.equal(head["stored"], head["w"].to(torch.bfloat16))
    net.params.mul_(0.5)
    net.pack_weights()
    assert torch.equal(head["stored"], head["w"].to(torch.bfloat16))


def test_fp32_and_logistic_stacks_keep_no_copies():
    owt()
    for dt, loss in (("f32", "softmax"), ("f32", "logistic"), ("bf16", "logistic")):
        assert new(4, 64, 64, 1, 10, dt, loss=loss).copies is None
