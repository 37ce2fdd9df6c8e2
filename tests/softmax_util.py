"""Softmax cross-entropy of a dense layer in 64 bits, and how far a call's results may be from it."""
import numpy as np
import torch

U = 2.0 ** -24          # half a step of fp32


def inputs(N, I, O, seed, dt="bf16", std=2.0, nobody=0.1, low=0, high=None):
    """Rows that point to their class, some hardly and some clearly; a share of rows without a class; weights of the rows."""
    g = np.random.default_rng(seed)
    high = O if high is None else high
    w = (g.standard_normal((O, I)) * std * I ** -0.5).astype(np.float32)
    labels = g.integers(low, high, N).astype(np.int32)
    x = (g.standard_normal((N, I)) + 2.0 * g.random((N, 1)) * w[labels % O]).astype(np.float32)
    labels = np.where(g.random(N) < nobody, g.choice([-1, -100, 1 << 30], N), labels).astype(np.int32)
    b = (g.standard_normal(O) * 0.3).astype(np.float32)
    weight = g.random(N).astype(np.float32)
    if dt == "bf16":
        x, w = (torch.from_numpy(a).bfloat16().float().numpy() for a in (x, w))
    return x, w, b, labels, weight


def planes_error(dt):
    """What is lost where an operand's value leaves as two: relative to the value (of a row whose values are alike in size)."""
    return 2.0 ** -17 if dt == "bf16" else 2.0 ** -21


class Reference:
    def __init__(self, x, w, b, labels, classes=None, off=0):
        with np.errstate(all="ignore"):
            self.x, self.w = x.astype(np.float64), w.astype(np.float64)
            self.b = np.zeros(len(w)) if b is None else b.astype(np.float64)
            classes = len(w) if classes is None else classes
            self.labels, self.off = labels, off
            self.real = (labels >= 0) & (labels < classes)
            self.x = np.where(self.real[:, None], self.x, 0.0)      # (a row without a class has no influence, whatever it holds)
            self.z = self.x @ self.w.T + self.b
            at = labels - off
            self.mine = self.real & (at >= 0) & (at < len(w))
            self.at = np.where(self.mine, at, 0)
            top = self.z.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0.0)
            self.lse = np.where(self.real, (top + np.log(np.exp(self.z - top).sum(1, keepdims=True)))[:, 0], 0.0)
            self.target = np.where(self.real, np.where(self.mine, self.z[np.arange(len(x)), self.at], -np.inf), 0.0)
            self.loss = np.where(self.real, np.where(np.isneginf(self.target), np.inf, self.lse - self.target), 0.0)

    def floors(self):
        """fp32 operands in two f16 values: a row's largest magnitude is at 2^14 or above, the second value's smallest step is 2^-24, half of it 2^-25: no value is off by
        more than 2^-39 of its row's largest, however small it is itself."""
        return tuple(np.abs(a).max(1, keepdims=True) for a in (self.x, self.w))

    def z_off(self):
        """How far an output may be off: operands in two f16 values lose 2^-22 of each (and the product of what is second, 2^-22), sums of I products and the
        bias in fp32, in any order and with each product or sum cut instead of rounded, 2 U a step."""
        size = np.abs(self.x) @ np.abs(self.w).T + np.where(np.isfinite(self.b), np.abs(self.b), 0.0)
        mx, mw = self.floors()
        floor = 2.0 ** -39 * (mx * np.abs(self.w).sum(1)[None, :] + np.abs(self.x).sum(1)[:, None] * mw.T)
        return (3 * 2.0 ** -22 + 2 * U * (self.x.shape[1] + 2)) * size + floor

    def lse_off(self):
        """The log of a sum of exponentials moves by no more than its largest argument does; each exponential is good to 2^-20 of itself (its argument, up to 87 in
        magnitude where it is not zero, is rounded: 87 U log2(e) < 2^-16.9 at the far end and 2^-20 of those that count), the sum in fp32 to U a step, of which a sum over
        O classes has O at most and no chain here is longer than 4096, and the result is rounded."""
        return self.z_off().max(1) + 2.0 ** -17 + U * min(self.z.shape[1], 4096) + 4 * U * np.abs(self.lse)

    def dz(self, lse, weight):
        with np.errstate(all="ignore"):
            p = np.where(np.isneginf(self.z), 0.0, np.exp(self.z - lse.astype(np.float64)[:, None]))
        d = p.copy()
        d[np.arange(len(d))[self.mine], self.at[self.mine]] -= 1.0
        f = np.where(self.real, 1.0 if weight is None else weight.astype(np.float64), 0.0)[:, None]
        # an output's error, the rounding of the difference and of the exponential itself, then of dz
        # (an exponential below 2^-126, the smallest normal number, and what is second of a value below 2^-117, may come out as zero: off by 2^-126 each)
        off = 2.0 ** -125 + p * np.expm1(self.z_off() + 2 * U * np.abs(lse)[:, None] + 2.0 ** -17) + 4 * U * np.abs(d)
        return d * f, off * np.abs(f)


def grads(ref, lse, weight, dt, alpha, beta, dw0, db0, little=False):
    """(dx, dw, db) and the bounds of their errors; little: of a small bf16 layer, dz in three values for dw (each rounding leaves 2^-8, the third 2^-24) and in two for dx."""
    dz, off = ref.dz(lse, weight)
    N, O = dz.shape
    second = planes_error(dt)
    aw, ax = np.abs(ref.w), np.abs(ref.x)
    one = 2.0 ** -8 if dt == "bf16" else second
    if little:
        second, one = 2.0 ** -24, 2.0 ** -16
    # dz in two f16 values is at 2^15 for 1 under one power of two: off by 2^-25 under it, 2^-40 without.  For dw a row n of dz comes times 2^-e, e of x's row, times the weight,
    # and the power of two is the largest such factor's or up to twice that; 2^-e is x's largest magnitude over 2^14 .. 2^15: the row's 2^-40 is that times the largest row's
    # weight times magnitude over this row's magnitude, times 4.  For dx the same with w's rows and no weight.  x and w have floors of their own.
    mx, mw = ref.floors()
    wt = np.where(ref.real, 1.0 if weight is None else np.abs(weight.astype(np.float64)), 0.0)[:, None]
    with np.errstate(all="ignore"):
        rx = np.where(mx > 0, 4 * (wt * mx).max(initial=0.0) / mx, 0.0)
        rw = np.where(mw > 0, 4 * mw.max() / mw, 0.0)
    low_x, low_w = 2.0 ** -40 * rx + 0 * ax, 2.0 ** -40 * rw + 0 * aw
    low_dw = (low_x * ax).sum(0)[None, :] + 2.0 ** -39 * (np.abs(dz).T @ (mx + 0 * ax)) if dt == "f32" else 0.0
    low_dx = wt * (low_w * aw).sum(0)[None, :] + 2.0 ** -39 * (np.abs(dz) @ (mw + 0 * aw)) if dt == "f32" else 0.0
    dx = dz @ ref.w
    dx_off = (off + np.abs(dz) * (one + second + 2 * U * (O + 2))) @ aw + np.abs(dx) * (2.0 ** -8 if dt == "bf16" else U) + low_dx
    dw = alpha * (dz.T @ ref.x) + (beta * dw0.astype(np.float64) if beta else 0.0)
    dw_off = abs(alpha) * ((off + np.abs(dz) * (2 * second + 2 * U * (N + 2))).T @ ax) + 4 * U * np.abs(dw) + (2 * U * np.abs(beta * dw0) if beta else 0.0) + abs(alpha) * low_dw
    db = alpha * dz.sum(0) + (beta * db0.astype(np.float64) if beta else 0.0)
    db_off = abs(alpha) * (off + np.abs(dz) * 2 * U * (N + 2)).sum(0) + 4 * U * np.abs(db) + (2 * U * np.abs(beta * db0) if beta else 0.0)
    return dict(dx=(dx, dx_off), dw=(dw, dw_off), db=(db, db_off))


def assert_within(got, want, off, what):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, what
    same = np.isfinite(want)
    assert np.array_equal(got[~same], want[~same], equal_nan=True), "%s: %r where %r" % (what, got[~same][:4], want[~same][:4])
    d = np.abs(got[same] - want[same])
    lim = (off if np.ndim(off) else np.full(want.shape, off))[same] + 2.0 ** -126
    bad = ~(d <= lim)
    assert not bad.any(), "%s: %d of %d off, the worst %.3g where %.3g is allowed" % (what, bad.sum(), bad.size, d[bad].max(), lim[bad][np.argmax(d[bad])])
    return float((d / lim).max()) if d.size else 0.0
