"""Rows in 8 bits whose threads one launch cannot count (2^32 and more): every row is written all the same, the ones about the ends of launches too.

The inputs repeat every PERIOD rows, so that the whole result is compared, exactly, with what the call gives for a few rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import owt  # noqa: E402

PERIOD = 251


def repeated(few, rows):
    return few.repeat((rows + PERIOD - 1) // PERIOD, *([1] * (few.dim() - 1)))[:rows].contiguous()


def same_in_every_row(whole, few):
    rows, at = whole.shape[0], 0
    step = PERIOD * (1 << 16)
    want = few.repeat(1 << 16, *([1] * (few.dim() - 1)))
    while at < rows:
        part = whole[at:at + step]
        assert torch.equal(part, want[:part.shape[0]]), at
        at += step


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_pack_and_norm():
    """32 threads a row of one value: 2^27 rows and three."""
    m = owt()
    rows = (1 << 27) + 3
    g = torch.Generator(device="cuda").manual_seed(4)
    x, r = (torch.randn((PERIOD, 1), generator=g, device="cuda") for _ in range(2))
    fq, fs, frstd, fh = torch.empty((PERIOD, 128), device="cuda", dtype=torch.int8), *(torch.empty(s, device="cuda") for s in ((PERIOD,), (PERIOD,), (PERIOD, 1)))
    q, s = torch.full((rows, 128), 99, device="cuda", dtype=torch.int8), torch.full((rows,), float("nan"), device="cuda")
    xs, rs = repeated(x, rows), repeated(r, rows)
    print("case pack", rows, flush=True)
    m.owt_q8_pack(PERIOD, 1, m.OWT_F32, x, fq, fs)
    m.owt_q8_pack(rows, 1, m.OWT_F32, xs, q, s)
    same_in_every_row(q, fq)
    same_in_every_row(s, fs)
    print("case norm", rows, flush=True)
    q.fill_(99)
    s.fill_(float("nan"))
    rstd, h = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows, 1), float("nan"), device="cuda")
    m.owt_rmsnorm_q8_fwd(PERIOD, 1, m.OWT_F32, x, r, None, 1e-5, fh, fq, fs, frstd)
    m.owt_rmsnorm_q8_fwd(rows, 1, m.OWT_F32, xs, rs, None, 1e-5, h, q, s, rstd)
    for whole, few in ((q, fq), (s, fs), (rstd, frstd), (h, fh)):
        same_in_every_row(whole, few)


def test_unpack():
    """128 threads a row of 65 pieces: 2^25 rows and one."""
    m = owt()
    rows, cols = (1 << 25) + 1, 257
    g = torch.Generator(device="cuda").manual_seed(5)
    fq = torch.randint(-127, 128, (PERIOD, m.owt_q8_pitch(cols)), generator=g, device="cuda", dtype=torch.int8)
    fs = torch.rand((PERIOD,), generator=g, device="cuda")
    q, s = repeated(fq, rows), repeated(fs, rows)
    few, x = torch.empty((PERIOD, cols), device="cuda"), torch.full((rows, cols), float("nan"), device="cuda")
    print("case unpack", rows, cols, flush=True)
    m.owt_q8_unpack(PERIOD, cols, m.OWT_F32, fq, fs, few)
    m.owt_q8_unpack(rows, cols, m.OWT_F32, q, s, x)
    same_in_every_row(x, few)
