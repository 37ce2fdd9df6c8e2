"""A launch counts its threads in 32 bits.  Products of more work-groups than that are refused before anything is launched (no device needed)."""
import pytest


@pytest.fixture(scope="module")
def m():
    import paper_1404_5997_amd as mod
    yield mod
    mod.owt_test_force_variant(-1, 0, 0)


class Scratch:
    """Stands for a large buffer: an address and a size, never read."""

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return 1 << 60

    def element_size(self):
        return 1


def refused(m, fn, *args):
    with pytest.raises(m.OwtError) as e:
        fn(*args)
    assert e.value.status == m.OWT_EUNSUPPORTED, str(e.value)


P = [256 * k for k in range(1, 7)]


# tiles of 64 x 64, 128 x 128 (256 threads) and 16 x 16 results (1024 threads): 2^24 and 2^22 work-groups and a few more
@pytest.mark.parametrize("tile,N,O", [(112, 1 << 18, (1 << 18) + 64), (111, 1 << 19, (1 << 19) + 128), (113, 1 << 15, (1 << 15) + 16), (112, 1 << 22, 1 << 22)])
def test_forward_products_of_too_many_tiles(m, tile, N, O):
    m.owt_test_force_variant(tile, 0, 0)
    refused(m, m.owt_fc_shard_q8_fwd, m.fc_desc(N, 64, O, 1), *P, None, 0)


# 32 x 128 results a work-group; the preparation's 64 x 64 values
@pytest.mark.parametrize("tile,N,I,O", [(114, 1 << 20, 131071, 1 << 10), (112, 1 << 18, 64, (1 << 18) + 64), (111, 1 << 22, 64, 1 << 22)])
def test_backward_passes_of_too_many_tiles(m, tile, N, I, O):
    m.owt_test_force_variant(tile, 0, 0)
    refused(m, m.owt_fc_shard_q8_bwd, m.fc_desc(N, I, O, 1), *P, 1.0, 0.0, 4096, 8192, None, Scratch(), 0)
