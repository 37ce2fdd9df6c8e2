"""Rows of 8-bit values, the RMS norm that writes them, and the dense shard on them, against plain implementations in 64 bits.

Tolerances are bounds of the arithmetic that the header states, taken element by element: fp32 roundings are 2^-24 of what is rounded
(U below), bf16 ones 2^-8 (8 bits kept), f16 ones 2^-11; a sum in fp32 of n terms is off by at most n U times the sum of their magnitudes.  Rows are compared with the
nearest whole number, from which the fp32 product of two rounded factors can be away by no more than 127 times its roundings."""
import sys

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import empty, force, owt, to_dev, to_host, workspace  # noqa: E402

U, UB = 2.0 ** -24, 2.0 ** -8


def say(*a):
    print(*a)
    sys.stdout.flush()


def code(m, dt):
    return m.OWT_BF16 if dt == "bf16" else m.OWT_F32


def stored(a, dt):
    return oracle.round_bf16(a) if dt == "bf16" else np.asarray(a, dtype=np.float32)


def rows_buffers(m, rows, cols):
    """Filled with what must not survive."""
    return torch.full((rows, m.owt_q8_pitch(cols)), 99, device="cuda", dtype=torch.int8), torch.full((rows,), float("nan"), device="cuda")


def host_rows(a):
    """8-bit rows and scales of a host array, padded: inputs of the shard's tests."""
    a = np.asarray(a, dtype=np.float64)
    amax = np.abs(a).max(1, keepdims=True)
    q = np.zeros((a.shape[0], owt().owt_q8_pitch(a.shape[1])), dtype=np.int8)
    q[:, :a.shape[1]] = np.rint(a * np.divide(127.0, amax, out=np.zeros_like(amax), where=amax > 0))
    return q, (amax / 127).astype(np.float32)[:, 0]


def check_rows(t, factor, q, scale, cols, rel, whole):
    """q, scale against the 8-bit rows of t (64 bits) times a factor a row: `rel` bounds the scale's error, `whole` q's beside the rounding."""
    amax = np.abs(t).max(1)
    np.testing.assert_array_equal(q[:, cols:], 0)
    assert np.all(np.abs(scale - amax / 127 * factor) <= rel * amax / 127 * np.abs(factor) + 1e-45)
    unit = np.where(amax > 0, 127 / np.where(amax > 0, amax, 1), 0)[:, None]
    assert np.all(np.abs(q[:, :cols] - t * unit) <= 0.5 + whole)
    assert np.all(np.abs(q).max(1)[amax > 0] == 127)


# one value, short of and past a piece and a row of 128 bytes, every launch shape, rows that are read twice
WIDTHS = [1, 3, 7, 16, 125, 128, 129, 250, 500, 1000, 1155, 2049, 4096, 5001, 9216, 16500]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cols", WIDTHS + [40000])
def test_pack_and_unpack(cols, dt):
    m = owt()
    rows = 37 if cols < 2000 else 3
    say("case pack", rows, cols, dt)
    g = np.random.default_rng(cols)
    x = stored(g.standard_normal((rows, cols)) * np.exp(g.uniform(-8, 8, (rows, 1))), dt)
    x[1] = 0.0
    x[2] = np.sign(x[2]) * np.float32(0.75)
    q, scale = rows_buffers(m, rows, cols)
    m.owt_q8_pack(rows, cols, code(m, dt), to_dev(x, dt), q, scale)
    back = torch.full((rows, cols), float("nan"), device="cuda", dtype=torch.bfloat16 if dt == "bf16" else torch.float32)
    m.owt_q8_unpack(rows, cols, code(m, dt), q, scale, back)
    torch.cuda.synchronize()
    qh, sh = to_host(q).astype(np.int64), to_host(scale)
    # x * (127 * (1 / max)): four roundings of a number up to 127
    check_rows(x.astype(np.float64), np.ones(rows), qh, sh.astype(np.float64), cols, U, 4 * 127 * U * 1.01)
    assert sh[1] == 0 and not qh[1].any()
    want = (qh[:, :cols].astype(np.float32) * sh[:, None])
    np.testing.assert_array_equal(to_host(back), stored(want, dt))


def test_pack_of_the_extremes():
    m = owt()
    tiny, huge = np.float32(1e-42), np.float32(3e38)
    x = np.array([[tiny, -tiny / 2, 0, tiny / 4], [huge, -huge / 2, 1, 0], [np.inf, 1, 2, 3], [1, np.nan, 2, np.inf], [-0.0, 0, -0.0, 0],
                  [2.0 ** -70, -2.0 ** -71, 0, 0], [2.0 ** -126, 2.0 ** -127, 0, 0]], dtype=np.float32)
    q, scale = rows_buffers(m, 7, 4)
    m.owt_q8_pack(7, 4, m.OWT_F32, to_dev(x), q, scale)
    back = torch.zeros((7, 4), device="cuda")
    m.owt_q8_unpack(7, 4, m.OWT_F32, q, scale, back)
    torch.cuda.synchronize()
    qh, b = to_host(q)[:, :4], to_host(back)
    assert np.isnan(b[2]).all() and np.isnan(b[3]).all() and not qh[2:5].any() and not b[4].any()
    for r in (0, 1, 5, 6):
        assert list(qh[r][:1]) == [127]
        # half a unit, and a scale that may be subnormal itself
        assert np.all(np.abs(b[r].astype(np.float64) - x[r]) <= 0.51 * np.abs(x[r]).max() / 127 + 127 * 1.5e-45)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("cols", WIDTHS)
def test_norm_forward(cols, residual, dt):
    m = owt()
    rows = 21 if cols < 2000 else 3
    say("case norm", rows, cols, dt, residual)
    g = np.random.default_rng(7000 + cols)
    x, r = (stored(g.standard_normal((rows, cols)) * s, dt) for s in (1.0, 3.0))
    gain = (1 + 0.3 * g.standard_normal(cols)).astype(np.float32)
    x[1] = r[1] = 0.0
    h32 = x + r if residual else x                                  # fp32, as the header says
    q, scale = rows_buffers(m, rows, cols)
    rstd, h = torch.full((rows,), float("nan"), device="cuda"), empty((rows, cols), dt) if residual else None
    m.owt_rmsnorm_q8_fwd(rows, cols, code(m, dt), to_dev(x, dt), to_dev(r, dt) if residual else None, to_dev(gain), 1e-5, h, q, scale, rstd)
    torch.cuda.synchronize()
    h64 = h32.astype(np.float64)
    want_rstd = 1 / np.sqrt((h64 * h64).mean(1) + np.float64(np.float32(1e-5)))
    n = min(cols, 64) + 24                                          # the longest chain of additions: a thread's, then a tree's
    got = to_host(rstd).astype(np.float64)
    assert np.all(np.abs(got - want_rstd) <= (n + 6) * U * want_rstd)
    # q: one rounding of t more than in a checkpoint, in the value and in the largest
    check_rows(h64 * gain, want_rstd, to_host(q).astype(np.int64), to_host(scale).astype(np.float64), cols, (n + 10) * U, 6 * 127 * U * 1.01)
    if residual:
        np.testing.assert_array_equal(to_host(h), stored(h32, dt))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("onto", ["x", "res"])
@pytest.mark.parametrize("cols", [125, 4096, 20000])
def test_norm_forward_in_place_without_gain(cols, onto, dt):
    m = owt()
    g = np.random.default_rng(cols)
    x, r = (stored(g.standard_normal((5, cols)), dt) for _ in range(2))
    outs = []
    for alias in (False, True):
        xd, rd = to_dev(x, dt), to_dev(r, dt)
        q, scale = rows_buffers(m, 5, cols)
        h = (xd if onto == "x" else rd) if alias else empty((5, cols), dt)
        m.owt_rmsnorm_q8_fwd(5, cols, code(m, dt), xd, rd, None, 0.0, h, q, scale)
        torch.cuda.synchronize()
        outs.append([to_host(t) for t in (h, q, scale)])
    for a, b in zip(*outs):
        np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(outs[0][0], stored(x + r, dt))


def norm_bwd_reference(dy, h, gain, rstd, dres):
    dy, h, gain, rstd = (np.asarray(a, dtype=np.float64) for a in (dy, h, gain, rstd))
    xn = h * rstd[:, None]
    gy = dy * gain
    mean = (gy * xn).mean(1, keepdims=True)
    size = np.abs(rstd)[:, None] * (np.abs(gy) + np.abs(xn) * np.abs(gy * xn).mean(1, keepdims=True))
    dh = rstd[:, None] * (gy - xn * mean)
    if dres is not None:
        dh, size = dh + dres, size + np.abs(dres)
    return dh, size, (dy * xn).sum(0), np.abs(dy * xn).sum(0)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 125), (70, 129), (5, 1000), (2100, 250), (1300, 2049), (33, 4096), (9, 9216), (3, 16500), (2, 32768)])
def test_norm_backward(rows, cols, dt):
    m = owt()
    say("case norm backward", rows, cols, dt)
    g = np.random.default_rng(rows * 31 + cols)
    dy, h, dres = (stored(g.standard_normal((rows, cols)), dt) for _ in range(3))
    gain = (1 + 0.3 * g.standard_normal(cols)).astype(np.float32)
    rstd = np.exp(g.uniform(-2, 2, rows)).astype(np.float32)
    dg0 = g.standard_normal(cols).astype(np.float32)
    ws = workspace(m.owt_rmsnorm_q8_workspace_bytes(rows, cols))
    for use_res, beta in ((False, 0.0), (True, -0.5)):
        dh = torch.full((rows, cols), float("nan"), device="cuda", dtype=torch.bfloat16 if dt == "bf16" else torch.float32)
        dgain = to_dev(dg0) if beta else torch.full((cols,), float("nan"), device="cuda")
        m.owt_rmsnorm_q8_bwd(rows, cols, code(m, dt), to_dev(dy, dt), to_dev(h, dt), to_dev(gain), to_dev(rstd), to_dev(dres, dt) if use_res else None,
                             0.25, beta, dh, dgain, ws)
        torch.cuda.synchronize()
        want, size, wg, wg_size = norm_bwd_reference(dy, h, gain, rstd, dres if use_res else None)
        n = min(cols, 64) + 24
        tol = (n + 10) * U * size + (UB * 1.01 * np.abs(want) if dt == "bf16" else 0)
        assert np.all(np.abs(to_host(dh) - want) <= tol)
        assert np.all(np.abs(to_host(dgain) - (0.25 * wg + beta * dg0)) <= (rows + 8) * U * (0.25 * wg_size + abs(beta) * np.abs(dg0)))


def test_norm_backward_in_place_without_gain_or_its_gradient():
    m = owt()
    g = np.random.default_rng(5)
    rows, cols = 40, 777
    dy, h, dres = (g.standard_normal((rows, cols)).astype(np.float32) for _ in range(3))
    rstd = np.ones(rows, dtype=np.float32)
    outs = []
    for onto in ("dy", "dres", None):
        dyd, dresd = to_dev(dy), to_dev(dres)
        dh = {"dy": dyd, "dres": dresd, None: empty((rows, cols))}[onto]
        m.owt_rmsnorm_q8_bwd(rows, cols, m.OWT_F32, dyd, to_dev(h), None, to_dev(rstd), dresd, 1.0, 0.0, dh, None)
        torch.cuda.synchronize()
        outs.append(to_host(dh))
    np.testing.assert_array_equal(outs[0], outs[2])
    np.testing.assert_array_equal(outs[1], outs[2])


def test_norm_gradient_against_differences():
    """The derivative of sum(w * norm(h)) in 64 bits by central differences: their error is h^2 times third derivatives, of order one here."""
    m = owt()
    g = np.random.default_rng(12)
    rows, cols, step = 3, 70, 1e-5
    h, w = g.standard_normal((rows, cols)).astype(np.float32), g.standard_normal((rows, cols)).astype(np.float32)
    gain = (1 + 0.3 * g.standard_normal(cols)).astype(np.float32)

    def loss(h64, g64):
        return (w * (h64 / np.sqrt((h64 * h64).mean(1, keepdims=True) + 1e-5) * g64)).sum()

    rstd = (1 / np.sqrt((h.astype(np.float64) ** 2).mean(1) + 1e-5)).astype(np.float32)
    dh, dgain = empty((rows, cols)), empty((cols,))
    m.owt_rmsnorm_q8_bwd(rows, cols, m.OWT_F32, to_dev(w), to_dev(h), to_dev(gain), to_dev(rstd), None, 1.0, 0.0, dh, dgain,
                         workspace(m.owt_rmsnorm_q8_workspace_bytes(rows, cols)))
    torch.cuda.synchronize()
    h64, g64 = h.astype(np.float64), gain.astype(np.float64)
    for r, c in [(0, 0), (1, 35), (2, 69), (2, 1)]:
        d = np.zeros_like(h64)
        d[r, c] = step
        assert abs((loss(h64 + d, g64) - loss(h64 - d, g64)) / (2 * step) - to_host(dh)[r, c]) < 1e-5
    for c in (0, 33, 69):
        d = np.zeros_like(g64)
        d[c] = step
        assert abs((loss(h64, g64 + d) - loss(h64, g64 - d)) / (2 * step) - to_host(dgain)[c]) < 1e-5


class Shard:
    def __init__(self, N, I, O, dt, bias=True, relu=True, seed=0):
        m = owt()
        self.N, self.I, self.O, self.dt, self.relu = N, I, O, dt, relu
        self.desc = m.fc_desc(N, I, 2 * O, 2, 1, code(m, dt), (m.OWT_BIAS if bias else 0) | (m.OWT_RELU if relu else 0))
        g = np.random.default_rng(seed + 1000 * N + 10 * I + O)
        self.xq, self.xs = host_rows(g.standard_normal((N, I)) * np.exp(g.uniform(-3, 3, (N, 1))))
        self.wq, self.ws = host_rows(g.standard_normal((O, I)) * 0.1 * np.exp(g.uniform(-1, 1, (O, 1))))
        self.b = (g.standard_normal(O) if bias else np.zeros(O)).astype(np.float32)
        self.dy = stored(g.standard_normal((N, O)) * np.exp(g.uniform(-6, 6, (N, 1))), dt)
        self.y = stored(np.maximum(g.standard_normal((N, O)), 0), dt)
        self.dw0, self.db0 = g.standard_normal((O, I)).astype(np.float32), g.standard_normal(O).astype(np.float32)

    def values(self):
        return self.xq[:, :self.I] * self.xs.astype(np.float64)[:, None], self.wq[:, :self.I] * self.ws.astype(np.float64)[:, None]

    def forward(self):
        m = owt()
        y = torch.full((self.N, self.O), float("nan"), device="cuda", dtype=torch.bfloat16 if self.dt == "bf16" else torch.float32)
        m.owt_fc_shard_q8_fwd(self.desc, to_dev(self.xq), to_dev(self.xs), to_dev(self.wq), to_dev(self.ws), to_dev(self.b), y,
                              workspace(m.owt_fc_shard_q8_workspace_bytes(self.desc, m.OWT_PASS_FWD)))
        torch.cuda.synchronize()
        return to_host(y)

    def check_forward(self):
        # (whole numbers first: sums that cancel to nothing do so only there)
        q = self.xq[:, :self.I].astype(np.float64) @ self.wq[:, :self.I].astype(np.float64).T
        prod = q * self.xs.astype(np.float64)[:, None] * self.ws
        want = prod + self.b
        # whole sum to fp32, product of the scales, their product, the bias
        tol = 4 * U * (np.abs(prod) + np.abs(want)) + 1e-37
        if self.relu:
            want = np.maximum(want, 0)
        if self.dt == "bf16":
            tol = tol + 1.01 * UB * np.abs(want)
        got = self.forward()
        assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / tol)

    def backward(self, alpha, beta, dx=True, db=True):
        m = owt()
        nan = float("nan")
        t = torch.bfloat16 if self.dt == "bf16" else torch.float32
        dxd = torch.full((self.N, self.I), nan, device="cuda", dtype=t) if dx else None
        dw = to_dev(self.dw0) if beta else torch.full((self.O, self.I), nan, device="cuda")
        dbd = (to_dev(self.db0) if beta else torch.full((self.O,), nan, device="cuda")) if db else None
        m.owt_fc_shard_q8_bwd(self.desc, to_dev(self.xq), to_dev(self.xs), to_dev(self.wq), to_dev(self.ws), to_dev(self.y, self.dt) if self.relu else None,
                              to_dev(self.dy, self.dt), alpha, beta, dxd, dw, dbd,
                              workspace(m.owt_fc_shard_q8_workspace_bytes(self.desc, m.OWT_PASS_BWD_DATA)))
        torch.cuda.synchronize()
        return to_host(dxd) if dx else None, to_host(dw), to_host(dbd) if db else None

    def check_backward(self, alpha=1.0, beta=0.0, dx=True, db=True):
        x, w = self.values()
        dz = np.where(self.y > 0, self.dy, 0).astype(np.float64) if self.relu else self.dy.astype(np.float64)
        gx, gw, gb = self.backward(alpha, beta, dx, db)

        def tolerance(a, b, row_max, length, planes):
            """a @ b: the product with the scale, two halves (or one), sums in fp32 of `planes` products for each term, 16 an instruction."""
            terms = np.abs(a) @ np.abs(b)
            parts = (2.0 ** -22 if planes == 2 else 2.0 ** -11) + U
            return (parts + (planes * length / 8 + 16) * 2 * U) * terms + 2.0 ** -38 * row_max * np.abs(b).sum(0) + 1e-37

        want = (dz.T @ x)
        tol = tolerance(dz.T * 1.0, x, np.abs(dz.T * self.xs).max(1)[:, None] / max(1e-30, self.xs.min() if self.xs.size else 1), self.N, 2)
        old = self.dw0.astype(np.float64)
        assert np.all(np.abs(gw - (alpha * want + beta * old)) <= abs(alpha) * tol + 4 * U * np.abs(beta * old))
        if db:
            assert np.all(np.abs(gb - (alpha * dz.sum(0) + beta * self.db0)) <= (self.N + 8) * U * (abs(alpha) * np.abs(dz).sum(0) + np.abs(beta * self.db0)))
        if dx:
            want = dz @ w
            tol = tolerance(dz, w, np.abs(dz * self.ws).max(1)[:, None] / self.ws.min(), self.O, 1 if self.dt == "bf16" else 2)
            assert np.all(np.abs(gx - want) <= tol + (1.01 * UB * np.abs(want) if self.dt == "bf16" else 0))


SHARDS = [(1, 1, 1), (1, 4096, 130), (2, 125, 33), (5, 640, 17), (16, 129, 512), (17, 300, 64), (63, 128, 65), (64, 127, 125), (65, 1000, 31),
          (128, 9216, 125), (300, 257, 190), (520, 90, 300), (40, 70, 3000), (1500, 40, 70)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", SHARDS)
def test_shard_forward(N, I, O, dt):
    say("case shard forward", N, I, O, dt)
    Shard(N, I, O, dt).check_forward()
    Shard(N, I, O, dt, bias=False, relu=False).check_forward()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", SHARDS)
def test_shard_backward(N, I, O, dt):
    say("case shard backward", N, I, O, dt)
    s = Shard(N, I, O, dt)
    s.y[0] = 0.0                                                    # a row that the mask leaves empty
    s.y[:, -1] = 0.0                                                # and a column
    s.check_backward(1.0 / N, 0.0)
    Shard(N, I, O, dt, relu=False).check_backward(0.5, -0.25, dx=N % 2 == 0, db=N % 3 == 0)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", [110, 111, 112])
def test_every_tile_and_split_of_the_products(tile, splits):
    say("case tile", tile, splits)
    with force(tile, splits):
        for N, I, O in ((300, 700, 520), (70, 1300, 33), (3, 260, 300)):
            Shard(N, I, O, "f32").check_forward()
            Shard(N, I, O, "bf16").check_backward(1.0, 0.5)
            Shard(N, I, O, "f32").check_backward()


@pytest.mark.parametrize("N,I,O", [(1, 1, 1), (1, 4096, 130), (16, 2500, 32), (3, 13000, 20), (17, 9216, 33), (65, 129, 31), (300, 700, 260)])
def test_the_forward_kernel_of_few_results(N, I, O):
    say("case few", N, I, O)
    with force(113):
        Shard(N, I, O, "f32").check_forward()
        Shard(N, I, O, "bf16", bias=False, relu=False).check_forward()


def test_shard_of_the_largest_sums():
    """Every product 127 * 127 (and 128 * 128, which rows of one's own may hold): sums just short of 2^31, exact in whole numbers."""
    m = owt()
    I = 131071
    for v in (127, -128):
        q = torch.zeros((2, m.owt_q8_pitch(I)), device="cuda", dtype=torch.int8)
        q[:, :I] = v
        one = torch.ones(2, device="cuda")
        y = torch.empty((2, 2), device="cuda")
        d = m.fc_desc(2, I, 2, 1)
        m.owt_fc_shard_q8_fwd(d, q, one, q, one, None, y, workspace(m.owt_fc_shard_q8_workspace_bytes(d, 0)))
        torch.cuda.synchronize()
        np.testing.assert_array_equal(to_host(y), np.float32(v * v * I))


def test_an_empty_batch():
    m = owt()
    for dt in ("f32", "bf16"):
        s = Shard(4, 50, 30, dt)
        d = m.fc_desc(0, 50, 30, 1, 0, code(m, dt), m.OWT_BIAS | m.OWT_RELU)
        m.owt_fc_shard_q8_fwd(d, None, None, to_dev(s.wq), to_dev(s.ws), to_dev(s.b), None)
        dw, db = to_dev(s.dw0), to_dev(s.db0)
        m.owt_fc_shard_q8_bwd(d, None, None, to_dev(s.wq), to_dev(s.ws), None, None, 1.0, 0.5, None, dw, db,
                              workspace(m.owt_fc_shard_q8_workspace_bytes(d, m.OWT_PASS_BWD_DATA)))
        m.owt_q8_pack(0, 50, code(m, dt), None, None, None)
        m.owt_q8_unpack(0, 50, code(m, dt), None, None, None)
        m.owt_rmsnorm_q8_fwd(0, 50, code(m, dt), None, None, None, 0.0, None, None, None)
        dgain = to_dev(s.db0)
        m.owt_rmsnorm_q8_bwd(0, 30, code(m, dt), None, None, None, None, None, 1.0, 2.0, None, dgain)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(to_host(dw), s.dw0 * np.float32(0.5))
        np.testing.assert_array_equal(to_host(db), s.db0 * np.float32(0.5))
        np.testing.assert_array_equal(to_host(dgain), s.db0 * np.float32(2))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_what_is_not_finite_goes_where_it_belongs(dt):
    """An infinite gradient in a masked place leaves no trace; one in an open place reaches its row of dx and its row of dw, and nothing else."""
    m = owt()
    s = Shard(70, 100, 90, dt)
    s.y[:] = 1.0
    s.y[3, 5] = s.y[4, 6] = 0.0
    s.dy[3, 5], s.dy[4, 6] = np.inf, np.nan
    s.check_backward()
    s.dy[10, 20] = np.inf
    gx, gw, gb = s.backward(1.0, 0.0)
    assert not np.isfinite(gx[10]).any() and not np.isfinite(gw[20]).any() and gb[20] == np.inf
    others = np.isfinite(np.delete(gx, 10, 0)).all() and np.isfinite(np.delete(gw, 20, 0)).all() and np.isfinite(np.delete(gb, 20)).all()
    assert others


def test_rows_beyond_32_bit_offsets():
    """The last rows of a checkpoint of more than 2^32 bytes."""
    m = owt()
    cols, rows = 32768, 140000
    q = torch.zeros((rows, cols), device="cuda", dtype=torch.int8)
    scale = torch.zeros((rows,), device="cuda")
    x = torch.zeros((rows, cols), device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-3:] = torch.randn((3, cols), generator=g, device="cuda").to(torch.bfloat16)
    m.owt_q8_pack(rows, cols, m.OWT_BF16, x, q, scale)
    few_q, few_s = rows_buffers(m, 3, cols)
    m.owt_q8_pack(3, cols, m.OWT_BF16, x[-3:].clone(), few_q, few_s)
    assert torch.equal(q[-3:], few_q) and torch.equal(scale[-3:], few_s) and not q[:-3].any() and not scale[:-3].any()
    m.owt_q8_unpack(rows, cols, m.OWT_BF16, q, scale, x)
    back = torch.empty((3, cols), device="cuda", dtype=torch.bfloat16)
    m.owt_q8_unpack(3, cols, m.OWT_BF16, few_q, few_s, back)
    assert torch.equal(x[-3:], back)
    # the shard's products on the same rows
    wq, ws = host_rows(np.random.default_rng(3).standard_normal((20, cols)))
    d, few = m.fc_desc(rows, cols, 20, 1), m.fc_desc(3, cols, 20, 1)
    y, y3 = torch.empty((rows, 20), device="cuda"), torch.empty((3, 20), device="cuda")
    wqd, wsd = to_dev(wq), to_dev(ws)
    m.owt_fc_shard_q8_fwd(d, q, scale, wqd, wsd, None, y, workspace(m.owt_fc_shard_q8_workspace_bytes(d, 0)))
    m.owt_fc_shard_q8_fwd(few, few_q, few_s, wqd, wsd, None, y3, workspace(m.owt_fc_shard_q8_workspace_bytes(few, 0)))
    torch.cuda.synchronize()
    assert torch.equal(y[-3:], y3) and not y[:-3].any()


def test_on_a_stream_of_its_own_and_in_a_graph():
    m = owt()
    s = Shard(40, 200, 60, "bf16")
    dev = [to_dev(a) for a in (s.xq, s.xs, s.wq, s.ws, s.b)]
    dy, yk = to_dev(s.dy, "bf16"), to_dev(s.y, "bf16")
    y, dx = empty((40, 60), "bf16"), empty((40, 200), "bf16")
    dw, db = empty((60, 200)), empty((60,))
    ws = workspace(max(m.owt_fc_shard_q8_workspace_bytes(s.desc, p) for p in (0, 1)))
    x = to_dev(stored(np.random.default_rng(1).standard_normal((40, 200)), "bf16"), "bf16")
    q, scale = rows_buffers(m, 40, 200)

    def step():
        m.owt_q8_pack(40, 200, m.OWT_BF16, x, q, scale)
        m.owt_fc_shard_q8_fwd(s.desc, q, scale, dev[2], dev[3], dev[4], y, ws)
        m.owt_fc_shard_q8_bwd(s.desc, q, scale, dev[2], dev[3], yk, dy, 1.0, 0.0, dx, dw, db, ws)

    step()
    torch.cuda.synchronize()
    want = [to_host(t) for t in (y, dx, dw, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    for a, b in zip((y, dx, dw, db), want):
        np.testing.assert_array_equal(to_host(a), b)
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for t in (y, dx, dw, db):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, dx, dw, db), want):
            np.testing.assert_array_equal(to_host(a), b)


# The pass in one launch splits dz times its scale in three bf16 parts (all 24 bits; two, 16 bits, for dx in bf16) and adds 16 terms of a part an
# instruction, 3 / 16 (2 / 16) of a rounding for a term: check_backward's bounds, of two halves and 2 / 8 (one half, 1 / 8), hold for it as well.
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(1, 1, 1), (2, 125, 33), (16, 129, 512), (17, 300, 64), (63, 128, 65), (65, 1000, 31), (128, 700, 125), (300, 257, 190),
                                   (40, 70, 2999)])
def test_the_backward_kernel_of_few_results(N, I, O, dt):
    say("case few, backward", N, I, O, dt)
    with force(114):
        s = Shard(N, I, O, dt)
        s.y[0] = 0.0
        s.y[:, -1] = 0.0
        s.check_backward(1.0 / N, 0.0)
        Shard(N, I, O, dt, relu=False).check_backward(0.5, -0.25, dx=N % 2 == 0, db=N % 3 == 0)


@pytest.mark.parametrize("tile", [111, 112])
def test_both_backward_products_in_one_launch(tile):
    say("case pair", tile)
    with force(tile):
        for N, I, O in ((1, 1, 1), (300, 700, 520), (70, 1300, 33), (3, 260, 300)):
            Shard(N, I, O, "bf16").check_backward(1.0, 0.5)
            Shard(N, I, O, "f32").check_backward()


def test_the_backward_kernel_of_few_results_keeps_what_is_not_finite_and_what_is_small():
    m = owt()
    with force(114):
        s = Shard(70, 100, 90, "f32")
        s.y[:] = 1.0
        s.y[3, 5] = 0.0
        s.dy[3, 5] = np.inf
        s.check_backward()
        s.dy[10, 20] = np.inf
        gx, gw, gb = s.backward(1.0, 0.0)
        assert not np.isfinite(gx[10]).any() and not np.isfinite(gw[20]).any() and gb[20] == np.inf
        assert np.isfinite(np.delete(gx, 10, 0)).all() and np.isfinite(np.delete(gw, 20, 0)).all()
        s = Shard(70, 100, 90, "f32", relu=False)
        s.dy *= np.float32(2.0 ** -60)                              # no row is helped by a power of two of its own
        s.check_backward()
        # an empty batch
        dw, db, d = torch.ones((3, 40), device="cuda"), torch.ones(3, device="cuda"), m.fc_desc(0, 40, 3, 1)
        wq, ws = torch.ones((3, 128), device="cuda", dtype=torch.int8), torch.ones(3, device="cuda")
        none = torch.empty(16, device="cuda")
        m.owt_fc_shard_q8_bwd(d, none, none, wq, ws, None, none, 1.0, 0.5, None, dw, db, workspace(m.owt_fc_shard_q8_workspace_bytes(d, m.OWT_PASS_BWD_DATA)))
        torch.cuda.synchronize()
        assert (to_host(dw) == 0.5).all() and (to_host(db) == 0.5).all()
