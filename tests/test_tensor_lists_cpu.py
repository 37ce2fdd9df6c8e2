"""Lists of tensors are of the type that a call asks for, not of its width alone (no device needed)."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def m():
    import paper_1404_5997_amd as mod
    return mod


@pytest.mark.parametrize("name,like", [("float16", "OWT_BF16"), ("int16", "OWT_BF16"), ("int32", "OWT_F32"), ("float64", "OWT_F32"), ("float64", "OWT_BF16")])
def test_values_of_another_type_are_refused(m, name, like):
    code = getattr(m, like)
    right = torch.float32 if code == m.OWT_F32 else torch.bfloat16
    new = lambda t: m.tensor_list([torch.zeros((k,), dtype=t) for k in (8, 12)])      # noqa: E731
    bad, ok, f32 = new(getattr(torch, name)), new(right), new(torch.float32)
    for call in (lambda: m.owt_grad_norm(bad, code, 256, None, 0), lambda: m.owt_grad_clip(bad, bad, code, 256, 1.0, 0), lambda: m.owt_grad_clip(ok, bad, code, 256, 1.0, 0),
                 lambda: m.owt_sgd_momentum_clipped(f32, bad, f32, 0.9, 0.1, 0.0, 1.0, 256, 1.0, None, 0),
                 lambda: m.owt_sgd_momentum_clipped(f32, f32, f32, 0.9, 0.1, 0.0, 1.0, 256, 1.0, bad, 0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        m.tensor_list([torch.zeros((4,), dtype=right), torch.zeros((4,), dtype=getattr(torch, name))])


def test_the_right_type_reaches_the_library(m):
    for code, t in ((m.OWT_F32, torch.float32), (m.OWT_BF16, torch.bfloat16)):
        lst = m.tensor_list([torch.zeros((8,), dtype=t)])
        with pytest.raises(m.OwtError):
            m.owt_grad_norm(lst, code, None, None, 0)           # no place for the norm
    with pytest.raises(m.OwtError):
        m.owt_grad_norm(m.tensor_list([]), 7, 256, None, 0)     # no such type
