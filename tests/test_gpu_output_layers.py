"""The output layers and the beam search on cuda:0 against the fp64 oracle.

Tolerances are error bounds of the formulas, per element, with u = 2^-24: a sum of n fp32
terms is within 2 n u of the sum of their magnitudes (2: additions may truncate), a bf16
result within 2^-8 of itself, expf-like functions within 2^-21. The search is exact.
"""
import math

import numpy as np
import pytest
import torch

from oracle import output_layers as ol
from paper_1904_03409_gb300 import binding as bd

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, FP = bd.SL_BF16, bd.SL_FP32
TYPES = pytest.mark.parametrize("dt", [FP, BF], ids=["fp32", "bf16"])


def tdt(dt):
    return torch.bfloat16 if dt == BF else torch.float32


def up(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def out(*s, dtype=torch.float32):
    t = torch.empty(*s, dtype=dtype, device="cuda")
    return t.fill_(float("nan")) if t.is_floating_point() else t.fill_(-77)


def f64(t):
    return t.double().cpu().numpy()


def within(got, want, tol, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(got - want)[bad].max()), np.argwhere(bad)[:3].tolist())


def rounded(rng, dt, *s, scale=1.0):
    """Values of the type, as fp64 and on the device."""
    t = torch.from_numpy(scale * rng.normal(size=s)).to(tdt(dt))
    return t.double().numpy(), t.cuda()


def out_tol(dt, want):
    return (2.0 ** -8 if dt == BF else 4 * U) * np.abs(want)


# ------------------------------------------------------------------ layer norm
@TYPES
@pytest.mark.parametrize("R,N", [(1, 1), (5, 100), (3, 8), (37, 33), (70, 200), (9, 257), (130, 1024), (11, 1025),
                                 (6, 2048), (5, 4099), (3, 8192), (2, 20001)])
def test_norm(dt, R, N):
    rng = np.random.default_rng(R * 7919 + N)
    x, xd = rounded(rng, dt, R, N, scale=0.7)
    gamma, beta = rng.normal(size=N).astype(np.float32), rng.normal(size=N).astype(np.float32)
    dy = rng.normal(size=(R, N)).astype(np.float32)
    eps = 1e-5
    op = bd.stacklstm_norm_create(R + 3, N, dt)
    y, mean, rstd = out(R, N, dtype=tdt(dt)), out(R), out(R)
    g, b = up(gamma), up(beta)
    bd.stacklstm_norm_forward(op, xd, g, b, eps, y, mean, rstd)
    wy, wm, wr = ol.norm_forward(x, gamma, beta, eps)
    big = np.abs(x).max(1, keepdims=True)
    n = 2 * U * (N + 16)
    within(mean, wm, n * big[:, 0], "mean")
    # the variance has the error of a sum of N squares and of the mean in them
    within(rstd, wr, wr * 2 * n * (1 + big[:, 0] * wr), "rstd")
    xh = (x - wm[:, None]) * wr[:, None]
    t_xh = n * (big * wr[:, None] + 2 * np.abs(xh) * (1 + big * wr[:, None])) + 8 * U * np.abs(xh)
    within(y, wy, t_xh * np.abs(gamma) + 4 * U * (np.abs(xh * gamma) + np.abs(beta)) + out_tol(dt, wy), "y")
    # the backward from the fp32 statistics
    m32, r32 = f64(mean), f64(rstd)
    dx, dg, db = out(R, N), out(N), out(N)
    dyd = up(dy)
    bd.stacklstm_norm_backward(op, dyd, xd, g, mean, rstd, dx, dg, db)
    wdx, wdg, wdb = ol.norm_backward(dy, x, gamma, m32, r32)
    xh = (x - m32[:, None]) * r32[:, None]
    a = dy * gamma.astype(np.float64)
    am, xm = np.abs(a).max(1, keepdims=True), np.abs(xh).max(1, keepdims=True)
    within(dx, wdx, r32[:, None] * n * (np.abs(a) + am + np.abs(xh) * am * xm) + 8 * U * np.abs(wdx), "dx")
    s = 2 * U * (R + 16)
    within(dg, wdg, s * np.abs(dy * xh).sum(0), "dgamma")
    within(db, wdb, s * np.abs(dy).sum(0), "dbeta")
    # again, without what may be left out, into the same bits
    dx2, y2 = out(R, N), out(R, N, dtype=tdt(dt))
    bd.stacklstm_norm_backward(op, dyd, xd, g, mean, rstd, dx2)
    bd.stacklstm_norm_forward(op, xd, g, b, eps, y2)
    assert torch.equal(dx, dx2) and torch.equal(y, y2)
    dg2 = out(N)
    bd.stacklstm_norm_backward(op, dyd, xd, g, mean, rstd, None, dg2)
    assert torch.equal(dg, dg2)
    # no weights: 1 and 0
    bd.stacklstm_norm_forward(op, xd, None, None, eps, y2)
    wy = ol.norm_forward(x, None, None, eps)[0]
    within(y2, wy, t_xh + 4 * U * np.abs(wy) + out_tol(dt, wy), "plain y")
    bd.stacklstm_op_status(op)


def test_norm_of_no_rows():
    op = bd.stacklstm_norm_create(4, 9, FP)
    e, dg, db = torch.empty(0, 9, device="cuda"), out(9), out(9)
    s = torch.empty(0, device="cuda")
    bd.stacklstm_norm_forward(op, e, None, None, 1e-5, e.clone())
    bd.stacklstm_norm_backward(op, e, e, None, s, s, None, dg, db)
    assert not dg.any() and not db.any()


def test_norm_gradient_is_that_of_differences():
    """dx against central differences of the kernel's own fp32 forward: the loss sum(y dy) changes
    by dx . v along v; at a step of 2^-7 the differences' own error (third derivatives, fp32
    rounding of y) stays below 2^-9 of the gradient's norm."""
    rng = np.random.default_rng(3)
    R, N = 4, 64
    x, dy, v = (rng.normal(size=(R, N)).astype(np.float32) for _ in range(3))
    op = bd.stacklstm_norm_create(R, N, FP)
    mean, rstd, y, dx = out(R), out(R), out(R, N), out(R, N)
    f = lambda a: (bd.stacklstm_norm_forward(op, up(a), None, None, 1e-5, y, mean, rstd), f64(y))[1]
    h = 2.0 ** -7
    diff = ((f(x + h * v) - f(x - h * v)) * dy).sum() / (2 * h)
    f(x)
    bd.stacklstm_norm_backward(op, up(dy), up(x), None, mean, rstd, dx)
    assert abs((f64(dx) * v).sum() - diff) <= 2.0 ** -9 * np.linalg.norm(f64(dx)) * np.linalg.norm(v)


# ------------------------------------------------------------------ linear layer
LINEAR = [(1, 1, 1), (1, 64, 40), (5, 100, 83), (8, 1024, 517), (17, 8, 300), (64, 200, 64), (65, 72, 130),
          (128, 64, 256), (130, 75, 100), (200, 333, 257), (300, 600, 200), (513, 48, 513), (1000, 128, 32),
          (2100, 520, 300), (66, 1100, 2500)]


@TYPES
@pytest.mark.parametrize("R,K,N", LINEAR)
@pytest.mark.parametrize("name", ["none", "gelu"])
def test_linear_forward(dt, R, K, N, name):
    linear_forward(dt, R, K, N, name)


@TYPES
@pytest.mark.parametrize("name", ["relu", "tanh", "silu"])
def test_linear_forward_activations(dt, name):
    linear_forward(dt, 70, 40, 90, name)


# sizes at which pairs of CTAs share a tile: of the forward, of dx and of dW, whole and ragged
WIDE = [(20001, 136, 330), (9001, 264, 330), (130, 2050, 5000), (300, 2048, 4000)]


@TYPES
@pytest.mark.parametrize("R,K,N", WIDE)
def test_linear_wide_tiles(dt, R, K, N):
    linear_forward(dt, R, K, N, "relu")
    linear_backward(dt, R, K, N, "none")


def linear_forward(dt, R, K, N, name):
    rng = np.random.default_rng(R + 31 * K + 977 * N)
    x, xd = rounded(rng, dt, R, K)
    W, Wd = rounded(rng, dt, N, K, scale=1 / math.sqrt(K))
    res, resd = rounded(rng, dt, R, N)
    bias = rng.normal(size=N).astype(np.float32)
    op = bd.stacklstm_linear_create(R + 2, K, N, dt, ol.ACTS.index(name))
    y, pre = out(R, N, dtype=tdt(dt)), out(R, N, dtype=tdt(dt))
    bd.stacklstm_linear_forward(op, xd, Wd, up(bias), resd, y, pre)
    bd.stacklstm_op_status(op)
    wy, wp = ol.linear_forward(x, W, bias, res, name)
    tol = 2 * U * (K + 16) * (np.abs(x) @ np.abs(W).T + np.abs(bias))
    within(pre, wp, tol + out_tol(dt, wp), "pre")
    # |act'| <= 1.13, the activation's own error is that of an expf-like function
    within(y, wy, 1.2 * tol + 2.0 ** -21 * (np.abs(wp) + 1) + out_tol(dt, wy) + 4 * U * np.abs(res), "y")
    y2 = out(R, N, dtype=tdt(dt))
    bd.stacklstm_linear_forward(op, xd, Wd, None, None, y2)
    w2, p2 = ol.linear_forward(x, W, None, None, name)
    within(y2, w2, 1.2 * tol + 2.0 ** -21 * (np.abs(p2) + 1) + out_tol(dt, w2), "bare y")
    # y in the place of the residual, the same bits
    bd.stacklstm_linear_forward(op, xd, Wd, up(bias), resd, resd)
    assert torch.equal(y, resd)


@TYPES
@pytest.mark.parametrize("R,K,N", LINEAR)
@pytest.mark.parametrize("name", ["none", "silu"])
def test_linear_backward(dt, R, K, N, name):
    linear_backward(dt, R, K, N, name)


@TYPES
@pytest.mark.parametrize("name", ["relu", "tanh", "gelu"])
def test_linear_backward_activations(dt, name):
    linear_backward(dt, 70, 40, 90, name)


def linear_backward(dt, R, K, N, name):
    rng = np.random.default_rng(R + 37 * K + 991 * N)
    x, xd = rounded(rng, dt, R, K)
    W, Wd = rounded(rng, dt, N, K, scale=1 / math.sqrt(K))
    pre, pred = rounded(rng, dt, R, N)
    dy, add = rng.normal(size=(R, N)).astype(np.float32), rng.normal(size=(R, K)).astype(np.float32)
    op = bd.stacklstm_linear_create(R, K, N, dt, ol.ACTS.index(name))
    dx, dW, db = out(R, K), out(N, K), out(N)
    p = pred if name != "none" else None
    dyd, addd = up(dy), up(add)
    bd.stacklstm_linear_backward(op, dyd, xd, Wd, p, addd, dx, dW, db)
    bd.stacklstm_op_status(op)
    wx, wW, wb, dz = ol.linear_backward(dy, x, W, pre, add, name)
    slack = 2.0 ** -20 * np.abs(dy) if name != "none" else 0 * np.abs(dy)  # of act'
    within(dx, wx, 2 * U * (N + 16) * (np.abs(dz) @ np.abs(W)) + slack @ np.abs(W) + 4 * U * (np.abs(add) + np.abs(wx)), "dx")
    within(dW, wW, 2 * U * (R + 16) * (np.abs(dz).T @ np.abs(x)) + slack.T @ np.abs(x), "dW")
    within(db, wb, 2 * U * (R + 16) * np.abs(dz).sum(0) + slack.sum(0), "dbias")
    # one at a time, the same bits; add in dx's own place
    dx2, dW2, db2 = addd.clone(), out(N, K), out(N)
    bd.stacklstm_linear_backward(op, dyd, None, Wd, p, dx2, dx2)
    bd.stacklstm_linear_backward(op, dyd, xd, None, p, None, None, dW2)
    bd.stacklstm_linear_backward(op, dyd, None, None, p, None, None, None, db2)
    assert torch.equal(dx, dx2) and torch.equal(dW, dW2) and torch.equal(db, db2)


@TYPES
def test_linear_of_no_rows_and_of_fewer(dt):
    op = bd.stacklstm_linear_create(300, 16, 24, dt)
    W = torch.ones(24, 16, device="cuda", dtype=tdt(dt))
    e = torch.empty(0, 16, device="cuda", dtype=tdt(dt))
    bd.stacklstm_linear_forward(op, e, W, None, None, torch.empty(0, 24, device="cuda", dtype=tdt(dt)))
    dW, db = out(24, 16), out(24)
    bd.stacklstm_linear_backward(op, torch.empty(0, 24, device="cuda"), e, W, None, None, None, dW, db)
    assert not dW.any() and not db.any()
    for r in (300, 2, 129):  # a handle takes any number of rows, in any order
        x = torch.ones(r, 16, device="cuda", dtype=tdt(dt))
        y = out(r, 24, dtype=tdt(dt))
        bd.stacklstm_linear_forward(op, x, W, None, None, y)
        assert y.eq(16).all()


def test_linear_fp32_values_of_every_scale():
    """The parts of an fp32 number cover its 24 bits at any exponent, and the largest ones."""
    x = np.array([[3.4028234e38, 0, 0], [0, 1 + 2.0 ** -23, 0], [0, 0, 2.0 ** -100 * (1 + 2.0 ** -20)], [0, -1 / 3, 0]], np.float32)
    op = bd.stacklstm_linear_create(4, 3, 3, FP)
    y = out(4, 3)
    bd.stacklstm_linear_forward(op, up(x), torch.eye(3, device="cuda"), None, None, y)
    assert np.array_equal(y.cpu().numpy(), x)


def test_linear_on_its_own_stream():
    rng = np.random.default_rng(0)
    st = torch.cuda.Stream()
    op = bd.stacklstm_linear_create(96, 40, 56, BF, stream=st)
    x, xd = rounded(rng, BF, 96, 40)
    W, Wd = rounded(rng, BF, 56, 40)
    y = out(96, 56, dtype=torch.bfloat16)
    st.wait_stream(torch.cuda.current_stream())
    bd.stacklstm_linear_forward(op, xd, Wd, None, None, y)
    bd.stacklstm_op_status(op)  # waits for its stream
    w = x @ W.T
    within(y, w, 2 * U * 56 * (np.abs(x) @ np.abs(W).T) + out_tol(BF, w))
    bd.stacklstm_op_set_stream(op, torch.cuda.current_stream())
    y2 = out(96, 56, dtype=torch.bfloat16)
    bd.stacklstm_linear_forward(op, xd, Wd, None, None, y2)
    assert torch.equal(y, y2)


@TYPES
@pytest.mark.parametrize("R,K,N", [(4, 200, 300), (300, 2000, 700)])
def test_linear_wait_that_runs_out_is_reported(dt, R, K, N, monkeypatch):
    """A wait budget of 0 cycles: the call ends, its status says so, and a handle with the usual
    budget works after it."""
    x, W = torch.ones(R, K, device="cuda", dtype=tdt(dt)), torch.ones(N, K, device="cuda", dtype=tdt(dt))
    y = out(R, N, dtype=tdt(dt))
    monkeypatch.setenv("STACKLSTM_WAIT_LIMIT_CYCLES", "0")
    op = bd.stacklstm_linear_create(R, K, N, dt)
    bd.stacklstm_linear_forward(op, x, W, None, None, y)
    with pytest.raises(bd.StackLSTMError) as e:
        bd.stacklstm_op_status(op)
    assert e.value.status == 6
    monkeypatch.delenv("STACKLSTM_WAIT_LIMIT_CYCLES")
    op = bd.stacklstm_linear_create(R, K, N, dt)
    bd.stacklstm_linear_forward(op, x, W, None, None, y)
    bd.stacklstm_op_status(op)
    assert y.eq(K).all()


# ------------------------------------------------------------------ distillation
def distill_case(rng, dt, R, V, k):
    z, zd = rounded(rng, dt, R, V, scale=2.0)
    idx = rng.integers(0, V, (R, k)).astype(np.int32)  # classes may repeat
    idx[rng.random((R, k)) < 0.2] = -1
    t = (2 * rng.normal(size=(R, k))).astype(np.float32)
    gold = rng.integers(-1, V, R).astype(np.int32)
    return z, zd, idx, t, gold


def distill_tol(z, idx, tau, alpha, scale, V):
    """Bounds of the loss and of the gradient from the sizes of what they are made of."""
    fin = np.where(np.isfinite(z), z, 0.0)
    span = np.abs(fin).max(1) * 2 + 1
    rel = 2 * U * (V / 32 + 64 + 4 * span * (1 / tau + 1)) + 2.0 ** -20
    amp = abs(scale) * (alpha * tau + 1 - alpha)
    tl = abs(scale) * (alpha * tau * tau + 1 - alpha) * (rel + 2.0 ** -19 * (span * (1 + 1 / tau) + math.log(V) + 8))
    return tl, rel[:, None] * amp


@TYPES
@pytest.mark.parametrize("R,V,k", [(1, 1, 1), (9, 2, 2), (33, 8, 3), (64, 83, 8), (10, 127, 5), (7, 1000, 33), (5, 1031, 64),
                                   (4, 4097, 256), (3, 9001, 7), (2, 33000, 32)])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.6), (0.7, 0.0)])
def test_distill(dt, R, V, k, tau, alpha):
    rng = np.random.default_rng(R * 31 + V + k)
    z, zd, idx, t, gold = distill_case(rng, dt, R, V, k)
    scale = 0.25
    op = bd.stacklstm_distill_create(R + 1, V, k, dt)
    loss, d = out(R), out(R, V)
    args = (zd, up(idx, torch.int32), up(t), up(gold, torch.int32), tau, alpha, scale)
    bd.stacklstm_distill_run(op, *args, loss, d)
    bd.stacklstm_op_status(op)
    wl, wd = ol.distill(z, idx, t, gold, tau, alpha, scale)
    tl, td = distill_tol(z, idx, tau, alpha, scale, V)
    within(loss, wl, tl, "loss")
    within(d, wd, td * 1.0, "dlogits")
    loss2, d2 = out(R), out(R, V)
    bd.stacklstm_distill_run(op, *args, None, d2)
    bd.stacklstm_distill_run(op, *args, loss2)
    assert torch.equal(d, d2) and torch.equal(loss, loss2)
    bd.stacklstm_distill_run(op, *args[:3], None, tau, alpha, scale, loss, d)  # no gold classes at all
    wl, wd = ol.distill(z, idx, t, None, tau, alpha, scale)
    within(loss, wl, tl, "loss without gold")
    within(d, wd, td, "dlogits without gold")


@TYPES
@pytest.mark.parametrize("V", [5, 90, 1500])
def test_distill_masks(dt, V):
    """Rows of -inf, classes of -inf with and without weight on them, the type's lowest value,
    absent teachers, teacher logits of -inf, padding."""
    rng = np.random.default_rng(V)
    R, k = 7, 4
    z, _, idx, t, gold = distill_case(rng, dt, R, V, k)
    low = float(torch.finfo(tdt(dt)).min)
    gold[:] = rng.integers(0, V, R)
    z[0] = -np.inf                                   # nothing to choose from
    z[1, :-1] = -np.inf                              # one class left
    idx[1], gold[1] = V - 1, V - 1
    z[2, ::2] = -np.inf                              # masked classes without weight
    idx[2], gold[2] = 1, 1
    z[3] = low                                       # every class masked by the lowest value: uniform
    idx[4], gold[4] = -1, -1                         # padding
    t[5] = -np.inf                                   # a teacher that says nothing
    t[6, 1:] = -np.inf                               # one entry left
    idx[6, 0] = 0
    zt = torch.from_numpy(z).to(tdt(dt))
    z = zt.double().numpy()
    op = bd.stacklstm_distill_create(R, V, k, dt)
    loss, d = out(R), out(R, V)
    bd.stacklstm_distill_run(op, zt.cuda(), up(idx, torch.int32), up(t), up(gold, torch.int32), 2.0, 0.5, 1.0, loss, d)
    bd.stacklstm_op_status(op)
    zz = np.where(z == low, 0.0, z)  # the oracle of a uniform row: any equal values
    zz[3] = 0.0
    wl, wd = ol.distill(zz, idx, t, gold, 2.0, 0.5, 1.0)
    tl, td = distill_tol(zz, idx, 2.0, 0.5, 1.0, V)
    within(loss, wl, tl)
    within(d, wd, td)
    assert not d[0].any() and loss[0] == 0 and not d[4].any() and loss[4] == 0


def test_distill_weight_on_a_masked_class_is_an_infinite_loss():
    z = torch.tensor([[0.0, -math.inf, 0.0]], device="cuda")
    op = bd.stacklstm_distill_create(1, 3, 1, FP)
    loss, d = out(1), out(1, 3)
    run = lambda idx, gold, alpha: bd.stacklstm_distill_run(op, z, up(np.array([[idx]]), torch.int32), torch.zeros(1, 1, device="cuda"),
                                                            up(np.array([gold]), torch.int32), 1.0, alpha, 1.0, loss, d)
    run(1, -1, 1.0)
    assert loss[0] == math.inf and d.tolist() == [[0.5, -1.0, 0.5]]
    run(-1, 1, 0.0)
    assert loss[0] == math.inf and d.tolist() == [[0.5, -1.0, 0.5]]


@TYPES
@pytest.mark.parametrize("V", [40, 3000])
def test_distill_nan_stays_in_its_row(dt, V):
    rng = np.random.default_rng(1)
    z, zd, idx, t, gold = distill_case(rng, dt, 3, V, 2)
    idx[:], gold[:] = 3, 4
    zd[1, 7] = float("nan")
    op = bd.stacklstm_distill_create(3, V, 2, dt)
    loss, d = out(3), out(3, V)
    bd.stacklstm_distill_run(op, zd, up(idx, torch.int32), up(t), up(gold, torch.int32), 1.0, 0.5, 1.0, loss, d)
    assert loss.isnan().tolist() == [False, True, False] and d.isnan().any(1).tolist() == [False, True, False]
    assert d[1].isnan().all()
    zd[1] = float("nan")
    bd.stacklstm_distill_run(op, zd, up(idx, torch.int32), up(t), up(gold, torch.int32), 1.0, 0.5, 1.0, loss, d)
    assert loss.isnan().tolist() == [False, True, False]


def test_distill_reports_bad_indices():
    op = bd.stacklstm_distill_create(2, 5, 2, FP)
    z, loss, d = torch.zeros(2, 5, device="cuda"), out(2), out(2, 5)
    t = torch.zeros(2, 2, device="cuda")
    idx = up(np.array([[0, 9], [1, -4]]), torch.int32)
    gold = up(np.array([5, 0]), torch.int32)
    bd.stacklstm_distill_run(op, z, idx, t, gold, 1.0, 0.5, 1.0, loss, d)
    with pytest.raises(bd.StackLSTMError) as e:
        bd.stacklstm_op_status(op)
    assert e.value.status == 1
    bd.stacklstm_op_status(op)  # cleared
    wl, wd = ol.distill(np.zeros((2, 5)), np.array([[0, -1], [1, -1]]), np.zeros((2, 2)), np.array([-1, 0]), 1.0, 0.5, 1.0)
    within(loss, wl, 1e-6)
    within(d, wd, 1e-6)


def test_distill_offsets_beyond_32_bits():
    """The last rows of logits with more than 2^32 elements."""
    V = 32003
    R = (1 << 32) // V + 7
    z = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    z[-1] = torch.arange(V, device="cuda").remainder(7).to(torch.bfloat16)
    d, loss = torch.empty(R, V, device="cuda"), out(R)
    idx = torch.full((R, 1), 3, dtype=torch.int32, device="cuda")
    op = bd.stacklstm_distill_create(R, V, 1, BF)
    bd.stacklstm_distill_run(op, z, idx, torch.zeros(R, 1, device="cuda"), None, 1.0, 1.0, 1.0, loss, d)
    zl = z[-2:].double().cpu().numpy()
    wl, wd = ol.distill(zl, np.full((2, 1), 3), np.zeros((2, 1)), None, 1.0, 1.0, 1.0)
    tl, td = distill_tol(zl, None, 1.0, 1.0, 1.0, V)
    within(loss[-2:], wl, tl)
    within(d[-2:], wd, td)
    within(d[:1], wd[:1], td[:1])


# ------------------------------------------------------------------ beam search
@TYPES
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 4, 7), (2, 8, 83), (1, 5, 1024), (2, 3, 1500), (1, 2, 40000), (2, 2, 70001)])
def test_lse(dt, B, K, V):
    rng = np.random.default_rng(V + K)
    z = 3 * rng.normal(size=(B, K, V))
    z[rng.random(z.shape) < 0.2] = -np.inf
    z[0, 0] = -np.inf
    zt = torch.from_numpy(z).to(tdt(dt))
    z = zt.double().numpy()
    op = bd.stacklstm_beam_create(B, K, V, 2, 8, dt)
    got = out(B, K)
    bd.stacklstm_beam_lse(op, zt.cuda(), got)
    want = ol.lse(z)
    g = f64(got)
    assert np.array_equal(np.isneginf(g), np.isneginf(want))
    fin = np.isfinite(want)
    span = np.abs(np.where(np.isfinite(z), z, 0)).max() + 1
    within(g[fin], want[fin], 2 * U * (V / 32 + 64 + 4 * span) + 2.0 ** -20 + 4 * U * span)


def select_both(dt, z, lse, score, done):
    """The kernel's choice and the oracle's, of values of the type."""
    zt = torch.from_numpy(np.ascontiguousarray(z)).to(tdt(dt))
    B, K, V = z.shape
    op = bd.stacklstm_beam_create(B, K, V, 2, 8, dt)
    want = ol.select(zt.float().numpy(), lse, score, done)
    for _ in range(2):  # the second call runs on what the first one left behind
        s, p, t = out(B, K), out(B, K, dtype=torch.int32), out(B, K, dtype=torch.int32)
        bd.stacklstm_beam_select(op, zt.cuda(), up(lse), up(score), up(done, torch.uint8), s, p, t)
        assert np.array_equal(s.cpu().numpy(), want[0])
        assert np.array_equal(p.cpu().numpy(), want[1])
        assert np.array_equal(t.cpu().numpy(), want[2])
    return want


@TYPES
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (2, 4, 1), (3, 2, 2), (2, 8, 83), (1, 64, 9), (2, 16, 511), (3, 5, 3333),
                                   (1, 8, 9001), (1, 64, 1031), (2, 1, 20000), (1, 40, 8192)])
def test_select(dt, B, K, V):
    rng = np.random.default_rng(B + K * 101 + V)
    z = rng.normal(size=(B, K, V))
    z[rng.random(z.shape) < 0.1] = -np.inf
    score = (-10 * rng.random((B, K))).astype(np.float32)
    done = (rng.random((B, K)) < 0.2).astype(np.uint8)
    lse = rng.normal(size=(B, K)).astype(np.float32)
    select_both(dt, z, lse, score, done)
    select_both(dt, z, None, score, None)


@TYPES
@pytest.mark.parametrize("K,V", [(4, 30), (8, 5000), (64, 700)])
def test_select_ties(dt, K, V):
    """Few distinct values, zeros of both signs: the lowest place first."""
    rng = np.random.default_rng(K)
    z = rng.integers(-2, 1, (2, K, V)).astype(np.float64)
    z[1] = 0.0
    z[1, :, ::3] = -0.0
    select_both(dt, z, None, np.zeros((2, K), np.float32), None)


@TYPES
@pytest.mark.parametrize("K,V", [(4, 3), (8, 4000)])
def test_select_runs_out_of_candidates(dt, K, V):
    """Fewer candidates than hypotheses, none at all, NaN, +inf, a normaliser of -inf."""
    z = np.full((4, K, V), -np.inf)
    z[0, 1, V // 2] = 1.0
    z[0, 2, 0] = 2.0
    z[2] = np.nan
    z[2, 3, 1] = -5.0
    z[3, 0, 2] = np.inf
    lse = np.zeros((4, K), np.float32)
    lse[0, 3] = -np.inf
    done = np.zeros((4, K), np.uint8)
    done[3, 1] = 1
    score = np.zeros((4, K), np.float32)
    want = select_both(dt, z, lse, score, done)
    assert (want[1][1] == -1).all() and want[1][0].tolist()[:3] == [2, 1, -1]
    score[:] = -np.inf  # the beam of an unused sentence
    assert (select_both(dt, z, lse, score, done)[1] == -1)[:2].all()


@TYPES
def test_select_all_the_best_in_one_place(dt):
    """Every one of the K best in one thread's reach, in neighbouring places, in one row."""
    K, V = 16, 9000
    for place in (lambda i: 3 + 256 * i, lambda i: 4000 + i, lambda i: V - K + i):
        z = np.full((1, K, V), -3.0)
        z[0, 5, [place(i) for i in range(K)]] = np.arange(K)
        select_both(dt, z, None, np.zeros((1, K), np.float32), None)


@TYPES
@pytest.mark.parametrize("B,K,S,H", [(1, 1, 1, 8), (2, 4, 5, 16), (3, 5, 70, 24), (2, 3, 9, 13), (1, 8, 130, 200), (2, 2, 4, 1)])
def test_reorder_and_push(dt, B, K, S, H):
    rng = np.random.default_rng(B + K + S + H)
    N = B * K
    h, hd = rounded(rng, dt, S, N, H)
    c, cd = rounded(rng, FP, S, N, H)
    old_h, ohd = rounded(rng, dt, S, N, H)
    old_c, ocd = rounded(rng, FP, S, N, H)
    parent = rng.integers(-1, K, (B, K)).astype(np.int32)
    p = rng.integers(0, S, N).astype(np.int32)
    op = bd.stacklstm_beam_create(B, K, 3, S, H, dt)
    po, th, tc = out(N, dtype=torch.int32), out(N, H, dtype=tdt(dt)), out(N, H)
    bd.stacklstm_beam_reorder(op, up(parent, torch.int32), up(p, torch.int32), hd, cd, po, ohd, ocd, th, tc)
    wp, wh, wc, wth, wtc = ol.reorder(parent, p, h, c, old_h, old_c)
    for got, want in ((po, wp), (ohd, wh), (ocd, wc), (th, wth), (tc, wtc)):
        assert np.array_equal(f64(got), want)
    bd.stacklstm_op_status(op)
    # a step on the result; what cannot be done is a hold and is reported
    ops = rng.integers(-1, 2, N).astype(np.int8)
    new_h, nhd = rounded(rng, dt, N, H)
    new_c, ncd = rounded(rng, FP, N, H)
    wp2, wh2, wc2, wth2, wtc2 = ol.push(ops, new_h, new_c, wp, wh, wc)
    bd.stacklstm_beam_push(op, up(ops, torch.int8), nhd, ncd, po, ohd, ocd, th, tc)
    for got, want in ((po, wp2), (ohd, wh2), (ocd, wc2), (th, wth2), (tc, wtc2)):
        assert np.array_equal(f64(got), want)
    under, over = ((ops == -1) & (wp == 0)).any(), ((ops == 1) & (wp == S - 1)).any()
    if under or over:
        with pytest.raises(bd.StackLSTMError) as e:
            bd.stacklstm_op_status(op)
        assert e.value.status in ((3,) if not over else (1,) if not under else (1, 3))
    else:
        bd.stacklstm_op_status(op)


def test_stack_calls_report_what_is_out_of_range():
    op = bd.stacklstm_beam_create(1, 2, 3, 4, 8, FP)
    h = torch.arange(4 * 2 * 8, device="cuda", dtype=torch.float32).view(4, 2, 8)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for parent, p in ((i32(7, 0), i32(1, 2)), (i32(0, 1), i32(9, -3)), (i32(-2, 0), i32(0, 0))):
        po, ho, co = out(2, dtype=torch.int32), torch.zeros_like(h), torch.zeros_like(h)
        bd.stacklstm_beam_reorder(op, parent.view(1, 2), p, h, h, po, ho, co)
        with pytest.raises(bd.StackLSTMError) as e:
            bd.stacklstm_op_status(op)
        assert e.value.status == 1
        assert po.ge(0).all() and po.lt(4).all()
    p = i32(1, 1)
    bd.stacklstm_beam_push(op, torch.tensor([5, 0], dtype=torch.int8, device="cuda"), h[0].clone(), h[0].clone(), p, h, h.clone())
    with pytest.raises(bd.StackLSTMError) as e:
        bd.stacklstm_op_status(op)
    assert e.value.status == 2 and p.tolist() == [1, 1]


def test_reorder_offsets_beyond_32_bits():
    """Stacks of more than 2^31 elements: the last slots of the last rows."""
    B, K, S, H = 128, 16, 1025, 1024
    N = B * K
    h = torch.empty(S, N, H, dtype=torch.bfloat16, device="cuda").normal_()
    c = torch.empty(S, N, H, device="cuda").normal_()
    ho, co = torch.zeros_like(h), torch.zeros_like(c)
    parent = torch.arange(K, dtype=torch.int32, device="cuda").flip(0).expand(B, K).contiguous()
    p = torch.zeros(N, dtype=torch.int32, device="cuda")
    p[-K:] = S - 1
    op = bd.stacklstm_beam_create(B, K, 3, S, H, BF)
    po = out(N, dtype=torch.int32)
    bd.stacklstm_beam_reorder(op, parent, p, h, c, po, ho, co)
    assert torch.equal(po, p)
    assert torch.equal(ho[:, -K:], h[:, -K:].flip(1)) and torch.equal(co[:, -K:], c[:, -K:].flip(1))
    assert torch.equal(ho[0], h[0].view(B, K, H).flip(1).reshape(N, H)) and not ho[1:, :-K].any()


# ------------------------------------------------------------------ alignment, refusals
def shifted(t):
    """The same values 16 bytes into another allocation: on 16 bytes, not on 32."""
    n = 16 // t.element_size()
    flat = torch.empty(t.numel() + n, dtype=t.dtype, device=t.device)
    flat[n:] = t.reshape(-1)
    return flat[n:].view(t.shape)


@TYPES
@pytest.mark.parametrize("N", [200, 1024, 83])
def test_tensors_on_16_bytes_give_the_same_bits(dt, N):
    rng = np.random.default_rng(N)
    R, k = 19, 5
    x, z = rounded(rng, dt, R, N)[1], rounded(rng, dt, R, N)[1]
    gamma, beta, dy = up(rng.normal(size=N)), up(rng.normal(size=N)), up(rng.normal(size=(R, N)))
    idx, t, gold = up(rng.integers(0, N, (R, k)), torch.int32), up(rng.normal(size=(R, k))), up(rng.integers(0, N, R), torch.int32)
    norm, lin, dist = (bd.stacklstm_norm_create(R, N, dt), bd.stacklstm_linear_create(R, N, 48, dt, bd.SL_ACT_SILU),
                       bd.stacklstm_distill_create(R, N, k, dt))
    W, dz, pre = rounded(rng, dt, 48, N)[1], up(rng.normal(size=(R, 48))), rounded(rng, dt, R, 48)[1]

    def run(f):
        o = [f(out(R, N, dtype=tdt(dt))), f(out(R)), f(out(R)), f(out(R, N)), f(out(N)), f(out(N)), f(out(R)), f(out(R, N)),
             f(out(R, 48, dtype=tdt(dt))), f(out(R, N)), f(out(48, N)), f(out(48))]
        bd.stacklstm_norm_forward(norm, f(x), f(gamma), f(beta), 1e-5, *o[:3])
        bd.stacklstm_norm_backward(norm, f(dy), f(x), f(gamma), o[1], o[2], *o[3:6])
        bd.stacklstm_distill_run(dist, f(z), f(idx), f(t), f(gold), 2.0, 0.5, 1.0, o[6], o[7])
        bd.stacklstm_linear_forward(lin, f(x), f(W), None, None, o[8])
        bd.stacklstm_linear_backward(lin, f(dz), f(x), f(W), f(pre), None, *o[9:])
        torch.cuda.synchronize()
        return o

    for a, b in zip(run(lambda v: v), run(shifted)):
        assert torch.equal(a, b)


def test_arguments_are_checked():
    norm, lin = bd.stacklstm_norm_create(4, 8, FP), bd.stacklstm_linear_create(4, 8, 8, FP, bd.SL_ACT_RELU)
    x, y = torch.zeros(4, 8, device="cuda"), out(4, 8)
    with pytest.raises(ValueError):  # more rows than the handle's
        bd.stacklstm_norm_forward(norm, torch.zeros(5, 8, device="cuda"), None, None, 1e-5, out(5, 8))
    with pytest.raises(ValueError):  # another type
        bd.stacklstm_norm_forward(norm, x.bfloat16(), None, None, 1e-5, y)
    with pytest.raises(ValueError):  # strides
        bd.stacklstm_norm_forward(norm, torch.zeros(8, 4, device="cuda").t(), None, None, 1e-5, y)
    with pytest.raises(ValueError):  # another shape
        bd.stacklstm_linear_forward(lin, x, torch.zeros(8, 9, device="cuda"), None, None, y)
    flat = torch.zeros(64, device="cuda")
    with pytest.raises(bd.StackLSTMError) as e:  # not on 16 bytes
        bd.stacklstm_norm_forward(norm, flat[1:33].view(4, 8), None, None, 1e-5, y)
    assert e.value.status == 1 and "aligned" in str(e.value)
    with pytest.raises(bd.StackLSTMError) as e:
        bd.stacklstm_norm_forward(norm, x, None, None, -1.0, y)
    assert e.value.status == 1
    with pytest.raises(bd.StackLSTMError) as e:  # relu's backward reads pre
        bd.stacklstm_linear_backward(lin, y, x, torch.zeros(8, 8, device="cuda"), None, None, out(4, 8))
    assert e.value.status == 1 and "pre" in str(e.value)
