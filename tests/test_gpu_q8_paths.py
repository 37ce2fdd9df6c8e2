"""The paths that serve large calls in 8 bits, at sizes of their own: which one a call takes is forced here, not left to the planner's costs.

110..112 are the products in tiles of 256, 128 and 64 behind their two launches of preparation, 113 the forward product of few results, 114 the backward
pass in one launch.  Tensors of more than 32 MB take variants that read or write past the caches: what they give is compared bit for bit with
what the same rows give in calls that are smaller than that."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import empty, force, owt, to_dev, to_host, workspace  # noqa: E402
from test_gpu_q8 import U, Shard, code, host_rows, rows_buffers, say, stored  # noqa: E402

PREPARED = [110, 111, 112]
BACKWARD = PREPARED + [114]
LARGE = 32 << 20
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dt])


def unwritten(shape, dt="f32"):
    return torch.full(shape, float("nan"), device="cuda", dtype=DT[dt])


# ---------------------------------------------------------------------------------------- backward pass of the shard


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kernel", BACKWARD)
def test_what_is_not_finite_goes_where_it_belongs(kernel, dt):
    """Masked infinities and NaN leave no trace; an open one reaches its row of dx and its row of dw, and nothing else."""
    say("case not finite", kernel, dt)
    with force(kernel):
        s = Shard(70, 100, 90, dt)
        s.y[:] = 1.0
        s.y[3, 5] = s.y[4, 6] = 0.0
        s.dy[3, 5], s.dy[4, 6] = np.inf, np.nan
        s.check_backward()
        for value in (np.inf, -np.inf, np.nan):
            s.dy[10, 20] = value
            gx, gw, gb = s.backward(1.0, 0.0)
            assert not np.isfinite(gx[10]).any() and not np.isfinite(gw[20]).any()
            np.testing.assert_equal(gb[20], np.float32(value))
            assert np.isfinite(np.delete(gx, 10, 0)).all() and np.isfinite(np.delete(gw, 20, 0)).all() and np.isfinite(np.delete(gb, 20)).all()
        # the values beside it keep their bits: what is not finite has no part in a row's power of two
        s.y[10, 20] = 0.0
        s.check_backward()
        # a column and a row with nothing finite in them, and one of zeros
        s.y[:] = 1.0
        s.dy[:, 7] = np.nan
        s.dy[12, :] = np.inf
        s.dy[:, 8] = 0.0
        s.dy[12, 8] = 0.0
        gx, gw, gb = s.backward(1.0, 0.0)
        assert not np.isfinite(gx).any(1).any() and not np.isfinite(gw[7]).any() and np.isnan(gb[7])       # (the column reaches every row of dx)
        assert not gw[8].any() and gb[8] == 0.0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("kernel", BACKWARD)
def test_without_dx_or_the_bias_gradient(kernel, relu, dt):
    say("case without", kernel, relu, dt)
    with force(kernel):
        for N, I, O in ((70, 129, 33), (300, 257, 190), (3, 40, 260)):
            s = Shard(N, I, O, dt, relu=relu)
            s.check_backward(1.0 / N, 0.0, dx=False)
            s.check_backward(0.5, -0.25, dx=False, db=False)
            s.check_backward(1.0, 0.0, db=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("kernel", BACKWARD)
def test_many_rows(kernel, relu, dt):
    """Strips of 192 rows and an end of 136: their sums and largest magnitudes are of several rounds of a work-group."""
    say("case many rows", kernel, relu, dt)
    with force(kernel):
        s = Shard(8200, 70, 41, dt, relu=relu)
        s.dy[5000:5200] *= np.float32(64)                           # the largest in one strip
        s.check_backward(1.0 / 8200, 0.0)
        s.check_backward(1.0, 0.5, dx=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kernel", BACKWARD)
def test_an_empty_batch(kernel, dt):
    m = owt()
    say("case empty", kernel, dt)
    with force(kernel):
        for I, O in ((50, 30), (300, 129)):
            g = np.random.default_rng(I)
            dw0, db0 = g.standard_normal((O, I)).astype(np.float32), g.standard_normal(O).astype(np.float32)
            wq, ws = host_rows(g.standard_normal((O, I)))
            d = m.fc_desc(0, I, O, 1, 0, code(m, dt), m.OWT_BIAS | m.OWT_RELU)
            scratch = workspace(m.owt_fc_shard_q8_workspace_bytes(d, m.OWT_PASS_BWD_DATA))
            for beta in (0.5, 0.0):
                dw, db = (to_dev(dw0), to_dev(db0)) if beta else (unwritten((O, I)), unwritten((O,)))
                m.owt_fc_shard_q8_bwd(d, None, None, to_dev(wq), to_dev(ws), None, None, 1.0, beta, None, dw, db, scratch)
                torch.cuda.synchronize()
                np.testing.assert_array_equal(to_host(dw), dw0 * np.float32(beta))
                np.testing.assert_array_equal(to_host(db), db0 * np.float32(beta))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("kernel", BACKWARD + [113])
def test_on_a_stream_of_its_own_and_in_a_graph(kernel, dt):
    m = owt()
    say("case stream and graph", kernel, dt)
    N, I, O = 90, 200, 60
    s = Shard(N, I, O, dt)
    wq, wsc, b = to_dev(s.wq), to_dev(s.ws), to_dev(s.b)
    dy, yk, x = to_dev(s.dy, dt), to_dev(s.y, dt), normal((N, I), dt, 1)
    y, dx, dw, db = empty((N, O), dt), empty((N, I), dt), empty((O, I)), empty((O,))
    q, scale = rows_buffers(m, N, I)
    with force(kernel):
        ws = workspace(max(m.owt_fc_shard_q8_workspace_bytes(s.desc, p) for p in (0, 1)))

        def step():
            m.owt_q8_pack(N, I, code(m, dt), x, q, scale)
            m.owt_fc_shard_q8_fwd(s.desc, q, scale, wq, wsc, b, y, ws)
            m.owt_fc_shard_q8_bwd(s.desc, q, scale, wq, wsc, yk, dy, 1.0, 0.0, dx, dw, db, ws)

        step()
        torch.cuda.synchronize()
        want = [to_host(t) for t in (y, dx, dw, db)]
        assert all(np.isfinite(a).all() for a in want)

        def check_anew(run):
            for t in (y, dx, dw, db):
                t.fill_(float("nan"))
            ws.fill_(255)
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            for a, b_ in zip((y, dx, dw, db), want):
                np.testing.assert_array_equal(to_host(a), b_)

        side = torch.cuda.Stream()

        def on_side():
            with torch.cuda.stream(side):
                step()

        check_anew(on_side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(4):
            check_anew(graph.replay)


# ---------------------------------------------------------------------------------------- tensors of more than 32 MB


def parts(rows, row_bytes):
    """Ranges of rows of a third of 32 MB."""
    each = LARGE // 3 // row_bytes
    return [(a, min(rows, a + each)) for a in range(0, rows, each)]


def large_rows(cols, e):
    return LARGE // (cols * e) + 5


# every number of threads a row, and rows that are read twice (more than 16384 fp32 values)
@pytest.mark.parametrize("dt,cols", [(dt, c) for dt in ("f32", "bf16") for c in (50, 125, 250, 500, 1000, 2049, 4096, 9216)] + [("f32", 16500), ("bf16", 32768)])
def test_large_norm_forward(cols, dt):
    m = owt()
    rows, e = large_rows(cols, 2 if dt == "bf16" else 4), 2 if dt == "bf16" else 4
    say("case large norm", rows, cols, dt)
    x, r, gain = normal((rows, cols), dt, 1), normal((rows, cols), dt, 2, 3.0), 1 + 0.3 * normal((cols,), "f32", 3)
    for residual in (True, False):
        want = []
        for a, b in parts(rows, cols * e):
            q, s = rows_buffers(m, b - a, cols)
            h, rstd = unwritten((b - a, cols), dt) if residual else None, unwritten((b - a,))
            m.owt_rmsnorm_q8_fwd(b - a, cols, code(m, dt), x[a:b].clone(), r[a:b].clone() if residual else None, gain, 1e-5, h, q, s, rstd)
            want.append((h, q, s, rstd))
        for onto in (None, "x", "res") if residual else (None,):
            xd, rd = x.clone(), r.clone() if residual else None
            h = {None: unwritten((rows, cols), dt) if residual else None, "x": xd, "res": rd}[onto]
            q, s = rows_buffers(m, rows, cols)
            rstd = unwritten((rows,))
            m.owt_rmsnorm_q8_fwd(rows, cols, code(m, dt), xd, rd, gain, 1e-5, h, q, s, rstd)
            for whole, few in zip((h, q, s, rstd), zip(*want)):
                assert whole is None or torch.equal(whole, torch.cat(few)), (residual, onto)
            if residual and onto != "x":
                assert torch.equal(xd, x)


@pytest.mark.parametrize("dt,cols", [(dt, c) for dt in ("f32", "bf16") for c in (125, 1000, 4096, 9216)] + [("f32", 40000), ("bf16", 40000)])
def test_large_pack(cols, dt):
    m = owt()
    rows, e = large_rows(cols, 2 if dt == "bf16" else 4), 2 if dt == "bf16" else 4
    say("case large pack", rows, cols, dt)
    x = normal((rows, cols), dt, 4)
    q, s = rows_buffers(m, rows, cols)
    m.owt_q8_pack(rows, cols, code(m, dt), x, q, s)
    for a, b in parts(rows, cols * e):
        fq, fs = rows_buffers(m, b - a, cols)
        m.owt_q8_pack(b - a, cols, code(m, dt), x[a:b].clone(), fq, fs)
        assert torch.equal(q[a:b], fq) and torch.equal(s[a:b], fs), (a, b)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [125, 500, 1000, 2049, 4096, 9216, 16500, 32768])
def test_large_norm_backward(cols, dt):
    m = owt()
    rows, e = large_rows(cols, 2 if dt == "bf16" else 4), 2 if dt == "bf16" else 4
    say("case large norm backward", rows, cols, dt)
    dy, h, dres = (normal((rows, cols), dt, 5 + k) for k in range(3))
    gain, rstd = 1 + 0.3 * normal((cols,), "f32", 8), 0.5 + normal((rows,), "f32", 9).abs()
    xn = h.double() * rstd.double()[:, None]
    want_dgain, size = (dy.double() * xn).sum(0), (dy.double() * xn).abs().sum(0)
    del xn
    scratch = workspace(m.owt_rmsnorm_q8_workspace_bytes(rows, cols))
    for residual in (True, False):
        want = []
        for a, b in parts(rows, cols * e):
            dh = unwritten((b - a, cols), dt)
            m.owt_rmsnorm_q8_bwd(b - a, cols, code(m, dt), dy[a:b].clone(), h[a:b].clone(), gain, rstd[a:b].clone(), dres[a:b].clone() if residual else None,
                                 1.0, 0.0, dh, None)
            want.append(dh)
        want = torch.cat(want)
        for onto in (None, "dy", "dres") if residual else (None, "dy"):
            dyd, dresd, dgain = dy.clone(), dres.clone() if residual else None, unwritten((cols,))
            dh = {None: unwritten((rows, cols), dt), "dy": dyd, "dres": dresd}[onto]
            m.owt_rmsnorm_q8_bwd(rows, cols, code(m, dt), dyd, h, gain, rstd, dresd, 1.0, 0.0, dh, dgain, scratch)
            assert torch.equal(dh, want), (residual, onto)
            assert bool(((dgain.double() - want_dgain).abs() <= (rows + 8) * U * size).all()), (residual, onto)


class Products:
    """Operands on the device; whole numbers, scales and gradients of a size."""

    def __init__(self, N, I, O, dt):
        m = owt()
        g = torch.Generator(device="cuda").manual_seed(N + I + O)
        self.N, self.I, self.O, self.dt = N, I, O, dt
        self.xq, self.wq = (self.rows(r, I, g) for r in (N, O))
        self.xs, self.ws = (torch.rand((r,), generator=g, device="cuda") + 0.1 for r in (N, O))
        self.b = normal((O,), "f32", 1)
        self.dy, self.y = normal((N, O), dt, 2), normal((N, O), dt, 3)
        self.m = m

    def rows(self, r, I, g):
        q = torch.randint(-127, 128, (r, owt().owt_q8_pitch(I)), generator=g, device="cuda", dtype=torch.int8)
        q[:, I:] = 0
        return q

    def desc(self, N, O):
        m = self.m
        return m.fc_desc(N, self.I, O, 1, 0, code(m, self.dt), m.OWT_BIAS | m.OWT_RELU)

    def forward(self, a, b):
        d, y = self.desc(b - a, self.O), unwritten((b - a, self.O), self.dt)
        self.m.owt_fc_shard_q8_fwd(d, self.xq[a:b].clone(), self.xs[a:b].clone(), self.wq, self.ws, self.b, y, workspace(self.m.owt_fc_shard_q8_workspace_bytes(d, 0)))
        return y

    def backward(self, rows, outs, beta=0.0):
        (a, b), (o, p) = rows, outs
        d, dx, db = self.desc(b - a, p - o), unwritten((b - a, self.I), self.dt), unwritten((p - o,))
        dw = unwritten((p - o, self.I)) if beta == 0 else torch.ones((p - o, self.I), device="cuda")
        if beta:
            db.fill_(1.0)
        self.m.owt_fc_shard_q8_bwd(d, self.xq[a:b].clone(), self.xs[a:b].clone(), self.wq[o:p].clone(), self.ws[o:p].clone(), self.y[a:b, o:p].contiguous().clone(),
                                   self.dy[a:b, o:p].contiguous().clone(), 0.5, beta, dx, dw, db, workspace(self.m.owt_fc_shard_q8_workspace_bytes(d, 1)))
        return dx, dw, db


# rows of whole fours (past the caches) and others
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("O", [4096, 4103])
@pytest.mark.parametrize("tile", PREPARED)
def test_large_results_of_the_forward_product(tile, O, dt):
    say("case large forward", tile, O, dt)
    p = Products(4099, 200, O, dt)
    assert p.N * O * (2 if dt == "bf16" else 4) > LARGE
    with force(tile):
        whole = p.forward(0, p.N)
        for a, b in parts(p.N, O * 4):
            assert torch.equal(whole[a:b], p.forward(a, b)), (a, b)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("I", [4096, 4103])
@pytest.mark.parametrize("tile", PREPARED)
def test_large_results_of_the_backward_products(tile, I, dt):
    """A row of dx depends on its row of dy alone, a row of dw on its column: either product in parts, the other one not looked at."""
    say("case large backward", tile, I, dt)
    with force(tile):
        p = Products(4099, I, 70, dt)
        assert p.N * I * (2 if dt == "bf16" else 4) > LARGE
        whole = p.backward((0, p.N), (0, p.O))[0]
        for a, b in parts(p.N, I * 4):
            assert torch.equal(whole[a:b], p.backward((a, b), (0, p.O))[0]), (a, b)
        p = Products(70, I, 4099, dt)
        for beta in (0.0, -0.5):
            _, dw, db = p.backward((0, p.N), (0, p.O), beta)
            for a, b in parts(p.O, I * 4):
                _, fw, fb = p.backward((0, p.N), (a, b), beta)
                assert torch.equal(dw[a:b], fw) and torch.equal(db[a:b], fb), (a, b, beta)
