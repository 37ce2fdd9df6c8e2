"""What softmax cross-entropy, the gradients' norm and the bounded update refuse before they touch a device."""
import pytest


@pytest.fixture(scope="module")
def m():
    import paper_1404_5997_amd as mod
    return mod


def refused(m, status, fn, *args, **kw):
    with pytest.raises(m.OwtError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)


def desc(m, **kw):
    g = dict(N=4, I=64, O_total=32, workers=1, rank=0, dtype=m.OWT_F32, flags=0)
    g.update(kw)
    return m.fc_desc(**g)


class Scratch:
    """Stands for device memory: an address and a size."""

    def __init__(self, n, at=1 << 20):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


def test_softmax_refuses_descriptors(m):
    p = [256 * k for k in range(1, 8)]
    for kw in (dict(N=-1), dict(I=0), dict(O_total=0), dict(O_total=33, workers=2), dict(workers=0), dict(rank=1), dict(rank=-1), dict(dtype=5), dict(flags=8),
               dict(flags=m.OWT_RELU), dict(flags=m.OWT_BIAS | m.OWT_RELU)):
        d = desc(m, **kw)
        refused(m, m.OWT_EINVAL, m.owt_fc_softmax_fwd, d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], Scratch(1 << 40), 0)
        refused(m, m.OWT_EINVAL, m.owt_fc_softmax_bwd, d, p[0], p[1], p[2], p[3], p[4], None, 1.0, 0.0, None, p[5], None, Scratch(1 << 40), 0)
        with pytest.raises(m.OwtError):
            m.owt_fc_softmax_workspace_bytes(d, 0)
    for kw in (dict(N=(1 << 22) + 1), dict(O_total=(1 << 22) + 1), dict(N=1 << 21, I=1024), dict(O_total=1 << 21, I=1024)):
        refused(m, m.OWT_EUNSUPPORTED, m.owt_fc_softmax_fwd, desc(m, **kw), p[0], p[1], p[2], p[3], p[4], None, None, Scratch(1 << 40), 0)
    for ps in (-1, 3):
        with pytest.raises(m.OwtError):
            m.owt_fc_softmax_workspace_bytes(desc(m), ps)


def test_softmax_refuses_pointers(m):
    p = [256 * k for k in range(1, 8)]
    d, big = desc(m, flags=m.OWT_BIAS), Scratch(1 << 40)
    ok = [p[0], p[1], p[2], p[3], p[4], p[5], p[6]]
    for at, bad in ((0, None), (1, None), (2, None), (4, None), (0, 260), (1, 264), (3, 257), (4, 258), (5, 260), (6, 268)):
        args = list(ok)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_fc_softmax_fwd, d, *args, big, 0)
    refused(m, m.OWT_EINVAL, m.owt_fc_softmax_fwd, d, p[0], p[1], p[2], None, p[4], p[5], None, big, 0)      # a target of no label
    refused(m, m.OWT_EINVAL, m.owt_fc_softmax_fwd, d, p[0], p[1], p[2], None, p[4], None, p[6], big, 0)
    two = desc(m, workers=2)
    refused(m, m.OWT_EINVAL, m.owt_fc_softmax_fwd, two, *ok, big, 0)                                           # a shard has no loss
    bwd = [p[0], p[1], p[2], p[3], p[4], p[5], 1.0, 0.0, p[6], 4096, 8192]
    for at, bad in ((0, None), (1, None), (2, None), (3, None), (4, None), (9, None), (0, 260), (3, 257), (4, 258), (5, 260), (8, 264), (9, 4100), (10, 8196),
                    (6, float("nan")), (7, float("inf"))):
        args = list(bwd)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_fc_softmax_bwd, d, *args, big, 0)


def test_softmax_refuses_scratch(m):
    p = [256 * k for k in range(1, 8)]
    for dt in (m.OWT_F32, m.OWT_BF16):
        d = desc(m, N=300, I=100, O_total=9000, dtype=dt)
        for ps in (0, 1):
            need = m.owt_fc_softmax_workspace_bytes(d, ps)
            assert need > 0 and need == m.owt_fc_softmax_workspace_bytes(d, ps)
            fwd = lambda ws: m.owt_fc_softmax_fwd(d, p[0], p[1], None, p[3], p[4], p[5], p[6], ws, 0)       # noqa: E731
            bwd = lambda ws: m.owt_fc_softmax_bwd(d, p[0], p[1], None, p[3], p[4], None, 1.0, 0.0, p[5], p[6], None, ws, 0)     # noqa: E731
            for ws in (None, Scratch(need - 1)):
                refused(m, m.OWT_EWORKSPACE, bwd if ps else fwd, ws)
            refused(m, m.OWT_EINVAL, bwd if ps else fwd, Scratch(need, (1 << 20) + 8))
            refused(m, m.OWT_EINVAL, bwd if ps else fwd, Scratch(need, 0))


def test_join_refuses(m):
    ok = [8, 4, 1000, 256, 512, 1024, 2048, 4096, 8192]
    for at, bad in ((0, 0), (1, -1), (2, 0), (3, None), (4, None), (5, None), (6, None), (3, 260), (6, 2052), (7, 4100), (8, 8196)):
        args = list(ok)
        args[at] = bad
        refused(m, m.OWT_EINVAL, m.owt_softmax_join, *args, 0)


def test_lists(m):
    torch = pytest.importorskip("torch")
    f = lambda *sizes: m.tensor_list([torch.zeros((k,)) for k in sizes])      # noqa: E731
    assert m.tensor_list([]).count == 0
    with pytest.raises(ValueError):
        m.tensor_list([torch.zeros((4, 8))[:, :4]])
    with pytest.raises(ValueError):
        m.tensor_list([torch.zeros((4,)), torch.zeros((4,), dtype=torch.bfloat16)])
    a, b, c = f(8, 12), f(8, 13), f(8)
    for bad in (b, c, m.tensor_list([torch.zeros((8,), dtype=torch.bfloat16), torch.zeros((12,), dtype=torch.bfloat16)])):
        with pytest.raises(ValueError):
            m.owt_grad_clip(a, bad, m.OWT_F32, 256, 1.0, 0)
        with pytest.raises(ValueError):
            m.owt_sgd_momentum_clipped(a, bad, a, 0.9, 0.1, 0.0, 1.0, 256, 1.0, None, 0)
        with pytest.raises(ValueError):
            m.owt_sgd_momentum_clipped(a, a, bad, 0.9, 0.1, 0.0, 1.0, 256, 1.0, None, 0)
    with pytest.raises(ValueError):
        m.owt_sgd_momentum_clipped(a, a, a, 0.9, 0.1, 0.0, 1.0, 256, 1.0, a, 0)      # a copy in bf16 is half as wide
    with pytest.raises(ValueError):
        m.owt_grad_norm(a, m.OWT_BF16, 256, None, 0)


class Fake:
    """A tensor of n values at an address, as a list keeps it."""

    def __init__(self, at, n, width=4):
        self.at, self.n, self.width = at, n, width

    def numel(self):
        return self.n

    def element_size(self):
        return self.width

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


def test_norm_clip_and_update_refuse(m):
    ok, odd, none = (m.tensor_list([Fake(at, 100), Fake(4096, 7)]) for at in (256, 260, 0))
    need = m.owt_grad_norm_workspace_bytes(ok)
    assert need > 0 and need == m.owt_grad_norm_workspace_bytes(ok)
    ws = Scratch(need)
    for bad in (odd, none):
        refused(m, m.OWT_EINVAL, m.owt_grad_norm, bad, m.OWT_F32, 512, ws, 0)
        refused(m, m.OWT_EINVAL, m.owt_grad_clip, bad, ok, m.OWT_F32, 512, 1.0, 0)
        refused(m, m.OWT_EINVAL, m.owt_grad_clip, ok, bad, m.OWT_F32, 512, 1.0, 0)
        for k in range(3):
            refused(m, m.OWT_EINVAL, m.owt_sgd_momentum_clipped, *[bad if j == k else ok for j in range(3)], 0.9, 0.1, 0.0, 1.0, 512, 1.0, None, 0)
        half = m.tensor_list([Fake(t.at, t.n, 2) for t in bad.tensors])
        refused(m, m.OWT_EINVAL, m.owt_sgd_momentum_clipped, ok, ok, ok, 0.9, 0.1, 0.0, 1.0, 512, 1.0, half, 0)
    for norm in (None, 516):
        refused(m, m.OWT_EINVAL, m.owt_grad_norm, ok, m.OWT_F32, norm, ws, 0)
        refused(m, m.OWT_EINVAL, m.owt_grad_clip, ok, ok, m.OWT_F32, norm, 1.0, 0)
        refused(m, m.OWT_EINVAL, m.owt_sgd_momentum_clipped, ok, ok, ok, 0.9, 0.1, 0.0, 1.0, norm, 1.0, None, 0)
    for most in (0.0, -1.0, float("nan")):
        refused(m, m.OWT_EINVAL, m.owt_grad_clip, ok, ok, m.OWT_F32, 512, most, 0)
        refused(m, m.OWT_EINVAL, m.owt_sgd_momentum_clipped, ok, ok, ok, 0.9, 0.1, 0.0, 1.0, 512, most, None, 0)
    for k in range(4):
        c = [0.9, 0.1, 0.0, 1.0]
        c[k] = float("inf")
        refused(m, m.OWT_EINVAL, m.owt_sgd_momentum_clipped, ok, ok, ok, *c, 512, 1.0, None, 0)
    for bad in (None, Scratch(need - 1)):
        refused(m, m.OWT_EWORKSPACE, m.owt_grad_norm, ok, m.OWT_F32, 512, bad, 0)
    refused(m, m.OWT_EINVAL, m.owt_grad_norm, ok, m.OWT_F32, 512, Scratch(need, (1 << 20) + 8), 0)
    huge = m.tensor_list([Fake(256, (1 << 40) + 1)])
    refused(m, m.OWT_EUNSUPPORTED, m.owt_grad_norm, huge, m.OWT_F32, 512, ws, 0)
    many = m.tensor_list([Fake(256, 1 << 40)] * 9)
    refused(m, m.OWT_EUNSUPPORTED, m.owt_grad_clip, many, many, m.OWT_F32, 512, 1.0, 0)
    with pytest.raises(m.OwtError):
        m.owt_grad_norm_workspace_bytes(huge)
