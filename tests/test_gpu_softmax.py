"""Softmax cross-entropy on a dense shard's outputs against the formulas in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from gpu_util import empty, owt, to_dev, to_host, workspace  # noqa: E402
from softmax_util import Reference, assert_within, grads, inputs  # noqa: E402

# rows, inputs, classes: one row, one class, sizes about tiles, steps and pieces, few rows of many classes, many rows of few
SIZES = [(1, 64, 1000), (1, 1, 1), (2, 3, 5), (7, 65, 33), (32, 128, 257), (33, 192, 256), (64, 64, 64), (65, 63, 129), (128, 256, 1000), (130, 1000, 125),
         (255, 130, 511), (256, 512, 512), (257, 72, 600), (300, 65, 4097), (515, 96, 10), (1000, 200, 2), (16, 2048, 3000), (3, 1537, 9001),
         (700, 640, 5000), (2100, 328, 3000)]


def code(dt):
    return owt().OWT_BF16 if dt == "bf16" else owt().OWT_F32


def run_fwd(N, I, O, dt, x, w, b, labels, workers=1, rank=0, want_loss=True):
    m = owt()
    d = m.fc_desc(N, I, O * workers, workers, rank, code(dt), m.OWT_BIAS if b is not None else 0)
    lse, target, loss = (torch.full((N,), float("nan"), device="cuda") for _ in range(3))
    m.owt_fc_softmax_fwd(d, to_dev(x, dt), to_dev(w, dt), to_dev(b), to_dev(labels), lse, target if labels is not None else None,
                         loss if want_loss else None, workspace(m.owt_fc_softmax_workspace_bytes(d, m.OWT_PASS_FWD)))
    torch.cuda.synchronize()
    return tuple(t.cpu().numpy() for t in (lse, target, loss))


def run_bwd(N, I, O, dt, x, w, b, labels, lse, weight, alpha, beta, dw0, db0, workers=1, rank=0, want_dx=True, want_db=True):
    m = owt()
    d = m.fc_desc(N, I, O * workers, workers, rank, code(dt), m.OWT_BIAS if b is not None else 0)
    dx = torch.full((N, I), float("nan"), device="cuda", dtype=torch.bfloat16 if dt == "bf16" else torch.float32) if want_dx else None
    dw = to_dev(dw0) if dw0 is not None else torch.full((O, I), float("nan"), device="cuda")
    db = (to_dev(db0) if db0 is not None else torch.full((O,), float("nan"), device="cuda")) if want_db else None
    m.owt_fc_softmax_bwd(d, to_dev(x, dt), to_dev(w, dt), to_dev(b), to_dev(labels), to_dev(lse), to_dev(weight), alpha, beta, dx, dw, db,
                         workspace(m.owt_fc_softmax_workspace_bytes(d, m.OWT_PASS_BWD_DATA)))
    torch.cuda.synchronize()
    return {k: to_host(t) for k, t in (("dx", dx), ("dw", dw), ("db", db)) if t is not None}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", SIZES)
def test_forward(N, I, O, dt):
    x, w, b, labels, _ = inputs(N, I, O, N + O, dt)
    ref = Reference(x, w, b, labels)
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    assert_within(target, ref.target, ref.z_off().max(1), "target")
    assert_within(loss, ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", SIZES)
def test_backward(N, I, O, dt):
    x, w, b, labels, weight = inputs(N, I, O, N + O + 1, dt)
    ref = Reference(x, w, b, labels)
    lse = ref.lse.astype(np.float32)
    g = np.random.default_rng(9)
    dw0, db0 = g.standard_normal((O, I)).astype(np.float32), g.standard_normal(O).astype(np.float32)
    # accumulated with the rows' weights, then written anew without
    for wt, alpha, beta, old in ((weight, 1.0 / N, 1.0, (dw0, db0)), (None, -0.5, 0.0, (None, None))):
        got = run_bwd(N, I, O, dt, x, w, b, labels, lse, wt, alpha, beta, *old)
        for k, (want, off) in grads(ref, lse, wt, dt, alpha, beta, dw0, db0).items():
            assert_within(got[k], want, off, "%s with beta %g" % (k, beta))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_what_is_not_wanted_is_left_out(dt):
    N, I, O = 70, 100, 300
    x, w, _, labels, _ = inputs(N, I, O, 4, dt)
    ref = Reference(x, w, None, labels)
    lse, _, _ = run_fwd(N, I, O, dt, x, w, None, None, want_loss=False)        # no labels: every row counts
    assert_within(lse, Reference(x, w, None, np.zeros_like(labels)).lse, Reference(x, w, None, np.zeros_like(labels)).lse_off(), "lse without labels")
    want = grads(ref, ref.lse.astype(np.float32), None, dt, 1.0, 0.0, None, None)
    for dx, db in ((True, False), (False, True), (False, False)):
        got = run_bwd(N, I, O, dt, x, w, None, labels, ref.lse.astype(np.float32), None, 1.0, 0.0, None, None, want_dx=dx, want_db=db)
        for k in got:
            assert_within(got[k], *want[k], k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(5, 40, 70), (300, 130, 520), (5, 64, 70), (300, 128, 520), (520, 64, 2000), (40, 2048, 96)])
def test_rows_without_a_class_have_no_influence(N, I, O, dt):
    x, w, b, labels, weight = inputs(N, I, O, 5, dt, nobody=0.3)
    labels[0], labels[-1] = -1, O
    ref = Reference(x, w, b, labels)
    for fill in (np.nan, np.inf, -np.inf):
        x[~ref.real] = fill
        lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
        assert_within(lse, ref.lse, ref.lse_off(), "lse")
        assert_within(loss, ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")
        assert (lse[~ref.real] == 0).all() and (target[~ref.real] == 0).all() and (loss[~ref.real] == 0).all()
        got = run_bwd(N, I, O, dt, x, w, b, labels, ref.lse.astype(np.float32), weight, 1.0, 0.0, None, None)
        for k, (want, off) in grads(ref, ref.lse.astype(np.float32), weight, dt, 1.0, 0.0, None, None).items():
            assert_within(got[k], want, off, k)
        assert (got["dx"][~ref.real] == 0).all()
    labels[:] = -1                          # nobody at all
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert not lse.any() and not target.any() and not loss.any()
    got = run_bwd(N, I, O, dt, x, w, b, labels, lse, weight, 1.0, 0.0, None, None)
    assert all(not v.any() for v in got.values())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(3, 40, 70), (270, 64, 600), (30, 2048, 130)])
def test_classes_that_are_taken_out(N, I, O, dt):
    x, w, b, labels, _ = inputs(N, I, O, 6, dt, nobody=0.0)
    b[1::3] = -np.inf
    ref = Reference(x, w, b, labels)
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    off = ref.z_off().max(1)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    assert_within(target, ref.target, off, "target")
    assert_within(loss, ref.loss, ref.lse_off() + off, "loss")
    got = run_bwd(N, I, O, dt, x, w, b, labels, ref.lse.astype(np.float32), None, 1.0, 0.0, None, None)
    for k, (want, o) in grads(ref, ref.lse.astype(np.float32), None, dt, 1.0, 0.0, None, None).items():
        assert_within(got[k], want, o, k)
    b[:] = -np.inf                          # nothing is left
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert (lse == -np.inf).all() and (target == -np.inf).all() and (loss == np.inf).all()
    got = run_bwd(N, I, O, dt, x, w, b, labels, lse, None, 1.0, 0.0, None, None)
    db = -np.bincount(labels, minlength=O).astype(np.float64)
    assert np.array_equal(got["db"], db)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_an_output_that_is_not_finite_reaches_its_row_alone(dt):
    N, I, O = 70, 72, 300
    x, w, b, labels, _ = inputs(N, I, O, 7, dt, nobody=0.0)
    x[3, 5] = np.nan
    x[60, 0] = np.inf
    clean = np.ones(N, bool)
    clean[[3, 60]] = False
    ref = Reference(np.where(clean[:, None], x, 0), w, b, labels)
    lse, _, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert not np.isfinite(lse[~clean]).any() and not np.isfinite(loss[~clean]).any()
    assert_within(lse[clean], ref.lse[clean], ref.lse_off()[clean], "lse")
    b[17] = np.inf                          # an infinite output: infinite sum, no gradient but of what is infinite
    lse, _, _ = run_fwd(N, I, O, dt, ref.x.astype(np.float32), w, b, labels)
    assert (lse == np.inf).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_large_and_small_outputs(dt):
    """Outputs of hundreds: exponentials far beyond fp32 on both sides."""
    N, I, O = 40, 128, 700
    x, w, b, labels, _ = inputs(N, I, O, 8, dt, std=90.0, nobody=0.0)
    b += 500.0
    ref = Reference(x, w, b, labels)
    lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    assert_within(loss, ref.loss, ref.lse_off() + ref.z_off().max(1) + 2.0 ** -24 * np.abs(ref.loss), "loss")
    got = run_bwd(N, I, O, dt, x, w, b, labels, ref.lse.astype(np.float32), None, 1.0, 0.0, None, None)
    for k, (want, off) in grads(ref, ref.lse.astype(np.float32), None, dt, 1.0, 0.0, None, None).items():
        assert_within(got[k], want, off, k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_shards_come_to_the_whole_layer(dt):
    N, I, O, K = 133, 100, 125, 8
    x, w, b, labels, weight = inputs(N, I, O * K, 10, dt)
    ref = Reference(x, w, b, labels)
    m = owt()
    lses, targets = torch.empty((K, N), device="cuda"), torch.empty((K, N), device="cuda")
    for k in range(K):
        part = slice(k * O, (k + 1) * O)
        l, t, _ = run_fwd(N, I, O, dt, x, w[part], b[part], labels, K, k, want_loss=False)
        share = Reference(x, w[part], b[part], labels, O * K, k * O)
        assert_within(t, share.target, share.z_off().max(1), "target of worker %d" % k)
        lses[k], targets[k] = torch.from_numpy(l).cuda(), torch.from_numpy(t).cuda()
    lse, target, loss = (torch.full((N,), float("nan"), device="cuda") for _ in range(3))
    m.owt_softmax_join(K, N, O * K, lses, targets, to_dev(labels), lse, target, loss)
    torch.cuda.synchronize()
    assert_within(lse.cpu().numpy(), ref.lse, ref.lse_off(), "lse")
    assert_within(target.cpu().numpy(), ref.target, ref.z_off().max(1), "target")
    assert_within(loss.cpu().numpy(), ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")
    l32 = ref.lse.astype(np.float32)
    want = grads(ref, l32, weight, dt, 1.0 / N, 0.0, None, None)
    dx = np.zeros((N, I))
    dx_off = np.zeros((N, I))
    for k in range(K):
        part = slice(k * O, (k + 1) * O)
        got = run_bwd(N, I, O, dt, x, w[part], b[part], labels, l32, weight, 1.0 / N, 0.0, None, None, K, k)
        assert_within(got["dw"], want["dw"][0][part], want["dw"][1][part], "dw")
        assert_within(got["db"], want["db"][0][part], want["db"][1][part], "db")
        dx += got["dx"]
        share = grads(Reference(x, w[part], b[part], labels, O * K, k * O), l32, weight, dt, 1.0, 0.0, None, None)["dx"]
        assert_within(got["dx"], *share, "dx of worker %d" % k)
        dx_off += share[1]
    assert_within(dx, want["dx"][0], dx_off, "dx")


def test_gradients_against_differences():
    N, I, O = 6, 20, 40
    x, w, b, labels, weight = inputs(N, I, O, 11, "f32")
    value = lambda x, w, b: (Reference(x, w, b, labels).loss * weight).sum()   # noqa: E731
    ref = Reference(x, w, b, labels)
    got = run_bwd(N, I, O, "f32", x, w, b, labels, ref.lse.astype(np.float32), weight, 1.0, 0.0, None, None)
    g, h = np.random.default_rng(1), 2.0 ** -13         # central differences in 64 bits: off by h^2 / 6 of the third derivative, some 1e-8
    for name, a, k in (("x", x, "dx"), ("w", w, "dw"), ("b", b, "db")):
        way = g.standard_normal(a.shape)
        ends = [value(*[v.astype(np.float64) + (s * h * way if n == name else 0.0) for n, v in (("x", x), ("w", w), ("b", b))]) for s in (1, -1)]
        along = (got[k] * way).sum()
        off = (grads(ref, ref.lse.astype(np.float32), weight, "f32", 1.0, 0.0, None, None)[k][1] * np.abs(way)).sum()
        assert abs(along - (ends[0] - ends[1]) / (2 * h)) <= off + 1e-6 * np.abs(way).sum(), name


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_an_empty_batch(dt):
    m = owt()
    d = m.fc_desc(0, 24, 50, 1, 0, code(dt), m.OWT_BIAS)
    assert m.owt_fc_softmax_workspace_bytes(d, m.OWT_PASS_FWD) == 0
    m.owt_fc_softmax_fwd(d, None, None, None, None, None)
    dw, db = torch.full((50, 24), 3.0, device="cuda"), torch.full((50,), 5.0, device="cuda")
    ws = workspace(m.owt_fc_softmax_workspace_bytes(d, m.OWT_PASS_BWD_DATA))
    m.owt_fc_softmax_bwd(d, None, None, None, None, None, None, 1.0, 0.5, None, dw, db, ws)
    torch.cuda.synchronize()
    assert (dw == 1.5).all() and (db == 2.5).all()
    m.owt_fc_softmax_bwd(d, None, None, None, None, None, None, 1.0, 0.0, None, dw, db, ws)
    torch.cuda.synchronize()
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(1, 200, 1000), (40, 96, 3000), (300, 130, 700)])
def test_the_same_call_gives_the_same_bits_and_writes_its_results_alone(N, I, O, dt):
    m = owt()
    x, w, b, labels, weight = inputs(N, I, O, 12, dt)
    d = m.fc_desc(N, I, O, 1, 0, code(dt), m.OWT_BIAS)
    X, W, B, L, WT = to_dev(x, dt), to_dev(w, dt), to_dev(b), to_dev(labels), to_dev(weight)
    need = [m.owt_fc_softmax_workspace_bytes(d, p) for p in (m.OWT_PASS_FWD, m.OWT_PASS_BWD_DATA)]
    pad, mark = 64, 77.0
    def around(shape, dtype=torch.float32):
        n = int(np.prod(shape))
        whole = torch.full((n + 2 * pad,), mark, device="cuda", dtype=dtype)
        return whole, whole[pad:pad + n].view(shape)
    t = torch.bfloat16 if dt == "bf16" else torch.float32
    first = None
    for fill in (0x00, 0xff, 0x55):          # whatever the scratch held, and not a byte behind it
        ws = [torch.full((n + 256,), fill, device="cuda", dtype=torch.uint8) for n in need]
        outs = [around(s, k) for s, k in (((N,), torch.float32), ((N,), torch.float32), ((N,), torch.float32), ((N, I), t), ((O, I), torch.float32), ((O,), torch.float32))]
        lse, target, loss, dx, dw, db = (o[1] for o in outs)
        m.owt_fc_softmax_fwd(d, X, W, B, L, lse, target, loss, ws[0][:need[0]])
        m.owt_fc_softmax_bwd(d, X, W, B, L, lse, WT, 1.0 / N, 0.0, dx, dw, db, ws[1][:need[1]])
        torch.cuda.synchronize()
        for whole, view in outs:
            n = view.numel()
            assert (whole[:pad] == mark).all() and (whole[pad + n:] == mark).all()
        assert all((a[n:] == fill).all() for a, n in zip(ws, need))
        got = [o[1].clone() for o in outs]
        if first is not None:
            assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(first, got))
        first = got


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N,I,O", [(16, 128, 2000), (300, 96, 700)])
def test_captured_and_replayed(N, I, O, dt):
    """Two graphs that share their scratch, replayed with new inputs and eager work between the replays."""
    m = owt()
    d = m.fc_desc(N, I, O, 1, 0, code(dt), m.OWT_BIAS)
    sets = [inputs(N, I, O, 20 + k, dt) for k in range(3)]
    X, W, B, L, WT = (to_dev(a, dt) if k < 2 else to_dev(a) for k, a in enumerate(sets[0]))
    need = max(m.owt_fc_softmax_workspace_bytes(d, p) for p in (0, 1))
    ws, ws2 = workspace(need), workspace(need)
    t = torch.bfloat16 if dt == "bf16" else torch.float32
    new = lambda: [torch.zeros(s, device="cuda", dtype=k) for s, k in (((N,), torch.float32), ((N,), torch.float32), ((N,), torch.float32), ((N, I), t), ((O, I), torch.float32), ((O,), torch.float32))]   # noqa: E731

    def fwd(o, w_):
        m.owt_fc_softmax_fwd(d, X, W, B, L, o[0], o[1], o[2], w_)

    def bwd(o, w_):
        m.owt_fc_softmax_bwd(d, X, W, B, L, o[0], WT, 1.0 / N, 0.0, o[3], o[4], o[5], w_)

    o, e = new(), new()
    fwd(e, ws2), bwd(e, ws2)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for g, f in zip(graphs, (fwd, bwd)):
            with torch.cuda.graph(g, stream=side):
                f(o, ws)
    torch.cuda.synchronize()
    for k in (0, 1, 2, 1):
        for a, b_ in zip((X, W, B, L, WT), sets[k]):
            a.copy_(to_dev(b_).to(a.dtype))
        for v in o:
            v.fill_(99)
        graphs[0].replay()
        graphs[1].replay()
        fwd(e, ws2), bwd(e, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(o, e)), k


def test_two_calls_at_once_on_streams_of_their_own():
    m = owt()
    N, I, O = 260, 256, 3000
    d = m.fc_desc(N, I, O, 1, 0, m.OWT_BF16, m.OWT_BIAS)
    need = m.owt_fc_softmax_workspace_bytes(d, 1)
    calls = []
    for k in range(2):
        x, w, b, labels, _ = inputs(N, I, O, 30 + k)
        lse = torch.from_numpy(Reference(x, w, b, labels).lse.astype(np.float32)).cuda()
        calls.append(dict(a=(to_dev(x, "bf16"), to_dev(w, "bf16"), to_dev(b), to_dev(labels), lse), ws=workspace(need), s=torch.cuda.Stream(),
                          o=[(empty((N, I), "bf16"), empty((O, I)), empty((O,))) for _ in range(2)]))
    torch.cuda.synchronize()
    for c in calls:
        m.owt_fc_softmax_bwd(d, *c["a"], None, 1.0, 0.0, *c["o"][0], c["ws"])
        torch.cuda.synchronize()
    for _ in range(3):
        for c in calls:
            m.owt_fc_softmax_bwd(d, *c["a"], None, 1.0, 0.0, *c["o"][1], c["ws"], stream=c["s"])
    torch.cuda.synchronize()
    for c in calls:
        assert all(torch.equal(p, q) for p, q in zip(*c["o"]))


# ------------------------------------------------------------------------------------------------ every tile, and sums that are split

TILES = {"256x256": 120, "128x128": 121, "128x128, two a CU": 122, "64x64": 123}


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("splits", [0, 1, 3])      # as planned (dx and dw then perhaps in one launch), none, three
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("N,I,O", [(5, 130, 70), (300, 256, 600), (520, 72, 1030), (129, 1024, 257)])
def test_tiles_and_splits(N, I, O, tile, splits, dt):
    from gpu_util import force
    x, w, b, labels, weight = inputs(N, I, O, N + I, dt)
    ref = Reference(x, w, b, labels)
    l32 = ref.lse.astype(np.float32)
    g = np.random.default_rng(3)
    dw0, db0 = g.standard_normal((O, I)).astype(np.float32), g.standard_normal(O).astype(np.float32)
    with force(TILES[tile], splits):
        lse, target, loss = run_fwd(N, I, O, dt, x, w, b, labels)
        got = run_bwd(N, I, O, dt, x, w, b, labels, l32, weight, 1.0 / N, 0.5, dw0, db0)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    assert_within(target, ref.target, ref.z_off().max(1), "target")
    assert_within(loss, ref.loss, ref.lse_off() + ref.z_off().max(1), "loss")
    for k, (want, off) in grads(ref, l32, weight, dt, 1.0 / N, 0.5, dw0, db0).items():
        assert_within(got[k], want, off, k)


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("N,I,O", [(520, 640, 1030), (1100, 512, 600), (130, 2100, 1000)])
def test_tiles_and_splits_of_larger_layers(N, I, O, tile, splits):
    test_tiles_and_splits(N, I, O, tile, splits, "bf16")


@pytest.mark.parametrize("N,I,O", [(1, 2048, 8300), (64, 300, 15000), (17, 4100, 4104)])
def test_dw_of_few_rows_keeps_all_of_dz(N, I, O):
    x, w, b, labels, weight = inputs(N, I, O, N + O + 3, "bf16")
    ref = Reference(x, w, b, labels)
    lse = ref.lse.astype(np.float32)
    got = run_bwd(N, I, O, "bf16", x, w, b, labels, lse, weight, 1.0 / N, 0.0, None, None)
    want = grads(ref, lse, weight, "bf16", 1.0 / N, 0.0, None, None)
    want["dw"] = grads(ref, lse, weight, "bf16", 1.0 / N, 0.0, None, None, little=True)["dw"]
    for k in want:
        assert_within(got[k], *want[k], k)


@pytest.mark.parametrize("tile", ["planned"] + list(TILES))
@pytest.mark.parametrize("N,I,O", [(1, 1, 1), (15, 384, 10), (65, 63, 129), (300, 130, 70), (128, 256, 1000), (900, 64, 300)])
def test_small_layers_keep_all_of_dz(N, I, O, tile):
    from gpu_util import force
    x, w, b, labels, weight = inputs(N, I, O, N + O + 2, "bf16")
    ref = Reference(x, w, b, labels)
    lse = ref.lse.astype(np.float32)
    with force(TILES.get(tile, -1), 0):
        got = run_bwd(N, I, O, "bf16", x, w, b, labels, lse, weight, 1.0 / N, 0.0, None, None)
    for k, (want, off) in grads(ref, lse, weight, "bf16", 1.0 / N, 0.0, None, None, little=True).items():
        assert_within(got[k], want, off, k)


FEW = 124              # few rows of fp32 with the weights as they lie


@pytest.mark.parametrize("N,I,O", [(1, 1, 1), (1, 1300, 70), (3, 5, 65), (16, 130, 257), (17, 33, 1000), (32, 256, 64), (40, 64, 300), (64, 259, 130), (48, 512, 1030),
                                   (5, 64, 16401), (20, 36, 17000), (64, 31, 16500), (33, 40, 9000), (60, 100, 8200)])
def test_few_rows(N, I, O):
    from gpu_util import force
    with force(FEW, 0):
        test_forward(N, I, O, "f32")
        test_backward(N, I, O, "f32")


def test_few_rows_with_all_that_may_be_in_them():
    from gpu_util import force
    with force(FEW, 0):
        for N, I, O in ((5, 40, 70), (40, 2048, 96), (64, 68, 520)):
            test_rows_without_a_class_have_no_influence(N, I, O, "f32")
            test_classes_that_are_taken_out(N, I, O, "f32")
            test_the_same_call_gives_the_same_bits_and_writes_its_results_alone(N, I, O, "f32")
        test_captured_and_replayed(16, 128, 2000, "f32")


@pytest.mark.parametrize("N,I,O", [(1, 2048, 4100), (16, 1024, 17000), (64, 1030, 5001)])
def test_few_rows_of_large_layers(N, I, O):
    test_forward(N, I, O, "f32")
    test_backward(N, I, O, "f32")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_pieces(dt):
    """So many rows that the classes are taken in pieces, the last of them short; few values of x, so that the reference is quick."""
    N, I, O = 20000, 8, 3000
    x, w, b, labels, weight = inputs(N, I, O, 40, dt)
    ref = Reference(x, w, b, labels)
    l32 = ref.lse.astype(np.float32)
    lse, _, _ = run_fwd(N, I, O, dt, x, w, b, labels)
    assert_within(lse, ref.lse, ref.lse_off(), "lse")
    got = run_bwd(N, I, O, dt, x, w, b, labels, l32, weight, 1.0 / N, 0.0, None, None)
    for k, (want, off) in grads(ref, l32, weight, dt, 1.0 / N, 0.0, None, None).items():
        assert_within(got[k], want, off, k)


def test_weights_of_more_than_four_gigabytes():
    """Offsets beyond 32 bits: rows at both ends and in the middle of 2 million classes."""
    m = owt()
    N, I, O = 3, 1024, 2_000_000
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty((O, I), device="cuda", dtype=torch.bfloat16).normal_(0.0, 2.0 * I ** -0.5, generator=g)
    x = torch.randn((N, I), generator=g, device="cuda").to(torch.bfloat16)
    labels = torch.tensor([O - 1, 0, O // 2], device="cuda", dtype=torch.int32)
    x = (x.float() + 4.0 * w[labels.long()].float()).to(torch.bfloat16)
    d = m.fc_desc(N, I, O, 1, 0, m.OWT_BF16, 0)
    lse, target, loss = (torch.empty((N,), device="cuda") for _ in range(3))
    ws = workspace(max(m.owt_fc_softmax_workspace_bytes(d, p) for p in (0, 1)))
    m.owt_fc_softmax_fwd(d, x, w, None, labels, lse, target, loss, ws)
    dx, dw, db = torch.empty((N, I), device="cuda", dtype=torch.bfloat16), torch.full((O, I), float("nan"), device="cuda"), torch.full((O,), float("nan"), device="cuda")
    m.owt_fc_softmax_bwd(d, x, w, None, labels, lse, None, 1.0, 0.0, dx, dw, db, ws)
    torch.cuda.synchronize()
    xd, dxr = x.double(), torch.zeros((N, I), device="cuda", dtype=torch.float64)
    z = torch.cat([xd @ w[k:k + 100_000].double().t().contiguous() for k in range(0, O, 100_000)], 1)
    want = torch.logsumexp(z, 1)
    size = (xd.abs() @ w[:1000].double().abs().t().contiguous()).max().item() * 1.5         # (sums of magnitudes hardly differ from row to row of w)
    off = 2.0 ** -23 * (I + 2) * size
    assert ((lse - want).abs() <= off + 2.0 ** -17 + 2.0 ** -12).all()
    assert ((target - z.gather(1, labels.long()[:, None])[:, 0]).abs() <= off).all()
    p = torch.exp(z - lse.double()[:, None])
    p.scatter_add_(1, labels.long()[:, None], torch.full((N, 1), -1.0, device="cuda", dtype=torch.float64))
    rel = 2 * off + 2.0 ** -16                   # of an exponential: its output's error, and the two bf16 values that it leaves as
    for k in range(0, O, 100_000):
        dxr += p[:, k:k + 100_000].contiguous() @ w[k:k + 100_000].double()
        wr = p[:, k:k + 100_000].t().contiguous() @ xd
        assert ((dw[k:k + 100_000].double() - wr).abs() <= rel * (p[:, k:k + 100_000].abs() + 2.0 ** -30).t().contiguous() @ xd.abs() + rel * 1e-4).all(), k
    assert ((db.double() - p.sum(0)).abs() <= rel * (p.abs().sum(0) + 1e-4)).all()
    assert ((dx.double() - dxr).norm() <= 2.0 ** -8 * 2 * dxr.norm())
