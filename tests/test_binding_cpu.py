"""What the binding takes where the library wants an address."""
import pytest


@pytest.fixture(scope="module")
def m():
    import paper_1404_5997_amd as mod
    return mod


class Address(int):
    """An address that notices when anything but a number is asked of it."""
    asked = 0

    def __getattr__(self, name):
        Address.asked += 1
        raise AttributeError(name)


def test_an_address_is_passed_on_without_being_taken_for_a_tensor(m):
    assert m._ptr(None) is None and m._ptr(4096) == 4096
    assert m._ptr(Address(512)) == 512 and Address.asked == 0


@pytest.mark.parametrize("what", [b"0123456789abcdef", "0123456789abcdef", bytearray(16), 4096.0, [4096], object()])
def test_what_is_no_tensor_and_no_address_is_refused(m, what):
    """Also where the call would not have looked at it: no rows, and bytes would go to the library as a pointer to host memory."""
    with pytest.raises((TypeError, AttributeError)):
        m._ptr(what)
    with pytest.raises((TypeError, AttributeError)):
        m.owt_q8_pack(0, 50, m.OWT_F32, what, None, None, 0)


def test_a_tensor_gives_its_address(m):
    torch = pytest.importorskip("torch")
    t = torch.zeros((4, 8))
    assert m._ptr(t) == t.data_ptr()
    with pytest.raises(ValueError):
        m._ptr(t[:, :4])
