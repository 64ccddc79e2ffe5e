"""What the output layers and the search meet at the edges of their ranges, on cuda:0: masks that
leave few classes, NaN before masked places, streams. Where a result has to be a given value or bit
pattern, equality is asked for."""
import math

import numpy as np
import pytest
import torch

import test_gpu_output_layers as base
from oracle import output_layers as ol
from paper_1904_03409_gb300 import binding as bd
from paper_1904_03409_gb300 import output_layers as om
from paper_1904_03409_gb300 import runner, workloads as wl

pytestmark = pytest.mark.gpu
BF, FP = bd.SL_BF16, bd.SL_FP32
TYPES = pytest.mark.parametrize("dt", [FP, BF], ids=["fp32", "bf16"])


def tdt(dt):
    return torch.bfloat16 if dt == BF else torch.float32


def up(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def out(*s, dtype=torch.float32):
    t = torch.empty(*s, dtype=dtype, device="cuda")
    return t.fill_(float("nan")) if t.is_floating_point() else t.fill_(-77)


# ------------------------------------------------------------------ selection
def select_is_exact(dt, z):
    """The kernel's choice and the oracle's, of values of the type."""
    B, K, V = z.shape
    zt = torch.from_numpy(z).to(tdt(dt))
    score = -np.arange(B * K, dtype=np.float32).reshape(B, K) / 8
    want = ol.select(zt.float().numpy(), None, score, None)
    op = bd.stacklstm_beam_create(B, K, V, 2, 8, dt)
    s, p, t = out(B, K), out(B, K, dtype=torch.int32), out(B, K, dtype=torch.int32)
    bd.stacklstm_beam_select(op, zt.cuda(), None, up(score), None, s, p, t)
    for got, w in zip((s, p, t), want):
        assert np.array_equal(got.cpu().numpy(), w)
    assert np.isfinite(want[0]).all()  # there are candidates enough


@TYPES
@pytest.mark.parametrize("K,V,allowed", [(64, 256, 40), (64, 128, 20), (40, 256, 36)])
def test_select_from_the_same_few_classes_of_every_hypothesis(dt, K, V, allowed):
    """More than 1024 candidates with fewer threads than hypotheses: all of those are ranked."""
    z = np.random.default_rng(K + V).normal(size=(1, K, V))
    z[:, :, allowed:] = -np.inf
    select_is_exact(dt, z)


@TYPES
@pytest.mark.parametrize("B,K,V,threads,allowed", [(1, 40, 8192, 256, 36), (7, 20, 32768, 512, 18)])
def test_select_from_classes_of_few_threads(dt, B, K, V, threads, allowed):
    """The same within a row: of the 16-byte pieces that a CTA's threads take in turn, those of a
    few threads."""
    E = 8 if dt == BF else 4
    z = np.random.default_rng(K + V).normal(size=(B, K, V))
    z[:, :, np.arange(V) // E % threads >= allowed] = -np.inf
    select_is_exact(dt, z)


# ------------------------------------------------------------------ distillation
@TYPES
@pytest.mark.parametrize("V", [40, 3000, 20000])
def test_distill_nan_before_masked_classes(dt, V):
    """A NaN stays in its row where every class after it is -inf."""
    rng = np.random.default_rng(V)
    R, k = 3, 2
    z = torch.from_numpy(rng.normal(size=(R, V))).to(tdt(dt))
    z[:, 16:] = -math.inf
    z[1, 7] = math.nan
    idx, gold = np.full((R, k), 3, np.int32), np.full(R, 4, np.int32)
    op = bd.stacklstm_distill_create(R, V, k, dt)
    loss, d = out(R), out(R, V)
    bd.stacklstm_distill_run(op, z.cuda(), up(idx, torch.int32), up(rng.normal(size=(R, k))), up(gold, torch.int32), 1.0, 0.5, 1.0,
                             loss, d)
    assert loss.isnan().tolist() == [False, True, False]
    assert d[1].isnan().all() and d[::2].isfinite().all()


# ------------------------------------------------------------------ the layers on a StackLSTM
def decoder(B=3, V=9, H=16, I=8, K=4):
    """Arguments of beam_decode up to the search's sizes."""
    rng = np.random.default_rng(11)
    f = lambda *s, sc=1.0: up((sc * rng.normal(size=s)).astype(np.float32))
    l = om.OutputLayers(B * K, H, V, 1, FP, seed=5)
    ops = torch.tensor([(1, 1, 1, -1, -1, 0, 0, 1, 0)[v % 9] for v in range(V)], dtype=torch.int8, device="cuda")
    return l, f(I + H, 4 * H, sc=0.4), f(4 * H, sc=0.2), f(V, I), ops, torch.tanh(f(B, H)), f(B, H)


def test_decode_on_another_stream_than_the_layers_were_made_on():
    """The same bits as on theirs, with that one busy at the call."""
    args = decoder()
    want = om.beam_decode(*args, 4, 6, 8)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(100_000_000)
    with torch.cuda.stream(side):
        got = om.beam_decode(*args, 4, 6, 8)
    torch.cuda.synchronize()
    again = om.beam_decode(*args, 4, 6, 8)
    for w, g, a in zip(want, got, again):
        assert torch.equal(w, g) and torch.equal(w, a)


@pytest.mark.parametrize("own,busy", [("side", "own"), ("side", "current"), ("default", "own")])
def test_train_step_of_a_stack_on_its_own_stream(own, busy):
    """The StackLSTM on a side stream, or it on the default one and the step called on a side
    stream: the same bits as on one, with either stream busy at the call."""
    T, B, H, V, k = 9, 12, 24, 37, 4
    w = wl.make_workload("streams", T=T, B=B, I=16, H=H, dtype="fp32", seed=3, ops_kind="random_walk", probs=(0.5, 0.3, 0.2),
                         bias_scale=0.2, h0_scale=0.5)
    rng = np.random.default_rng(4)
    teacher = (up(rng.integers(-1, V, (T * B, k)), torch.int32), up(rng.normal(size=(T * B, k))),
               up(rng.integers(-1, V, T * B), torch.int32))
    results = []
    default, side = torch.cuda.default_stream(), torch.cuda.Stream()
    for stack, current in ((default, default), (side, default) if own == "side" else (default, side)):
        hd = bd.stacklstm_create(T, B, 16, H, FP, 0, stack)
        bd.stacklstm_set_async(hd, True)
        with torch.cuda.stream(current):
            layers = om.OutputLayers(T * B, H, V, k, FP, seed=7)
        torch.cuda.synchronize()
        ins, o = runner.upload(w), runner.alloc_outputs(w)
        for t in (*o.values(), *layers.grads.values()):
            t.fill_(math.nan if t.is_floating_point() else 0)
        x = ins["x"]
        ins["x"] = torch.zeros_like(x)
        torch.cuda.synchronize()
        if stack is not current:
            with torch.cuda.stream(stack if busy == "own" else current):
                torch.cuda._sleep(100_000_000)
        with torch.cuda.stream(current):
            ins["x"].copy_(x)  # an input that the current stream's work writes
            loss = om.train_step(hd, ins, o, layers, *teacher)
            results.append([loss.clone(), *(layers.grads[n].clone() for n in sorted(layers.grads)),
                            *(o[n].clone() for n in ("y", "dx", "dh0", "dc0", "dW", "dbias"))])
        torch.cuda.synchronize()
        layers.status()
        bd.stacklstm_status(hd)
        hd.destroy()
        layers.destroy()
    for a, b in zip(*results):
        assert torch.equal(a, b) and a.isfinite().all()


def test_decode_reports_what_its_layers_detected(monkeypatch):
    """A wait of the layers' contractions that runs out (a budget of 0 cycles)."""
    monkeypatch.setenv("STACKLSTM_WAIT_LIMIT_CYCLES", "0")
    args = decoder()
    monkeypatch.delenv("STACKLSTM_WAIT_LIMIT_CYCLES")
    with pytest.raises(bd.StackLSTMError) as e:
        om.beam_decode(*args, 4, 2, 8)
    assert e.value.status == 6
    args[0].status()  # cleared


def test_decode_hypotheses_that_run_out_have_no_classes():
    """Two classes, an end and a pop, on empty stacks: one sequence, the end alone."""
    layers, W, bias, emb, _, h0, c0 = decoder(B=2, V=2, K=4)
    ops = torch.tensor([0, -1], dtype=torch.int8, device="cuda")
    score, seqs = om.beam_decode(layers, W, bias, emb, ops, h0, c0, 4, 3, 0)
    assert score.isfinite().tolist() == [[True, False, False, False]] * 2
    assert seqs.tolist() == [[[0, -1, -1]] + [[-1, -1, -1]] * 3] * 2


def test_learn_of_no_rows():
    """Zero gradients, not an error."""
    layers = om.OutputLayers(4, 16, 9, 2, BF)
    e = lambda *s, dtype=torch.float32: torch.empty(0, *s, dtype=dtype, device="cuda")
    for g in layers.grads.values():
        g.fill_(math.nan)
    loss, dy = layers.learn(e(16, dtype=torch.bfloat16), e(2, dtype=torch.int32), e(2), e(dtype=torch.int32))
    layers.status()
    assert loss.shape == (0,) and dy.shape == (0, 16)
    assert all(not g.any() for g in layers.grads.values())


# ------------------------------------------------------------------ normalisers
@TYPES
@pytest.mark.parametrize("V", [5, 83, 1500, 9001, 40000, 70001])
def test_lse_of_infinite_logits(dt, V):
    """+inf is a row's normaliser, -inf that of a row without classes, NaN stays."""
    rng = np.random.default_rng(V)
    z = torch.from_numpy(rng.normal(size=(1, 6, V))).to(tdt(dt)).cuda()
    z[0, 0, V // 2] = math.inf
    z[0, 1] = -math.inf
    z[0, 1, V - 1] = math.inf
    z[0, 2] = math.inf
    z[0, 3] = -math.inf
    z[0, 4, 0], z[0, 4, V - 1] = math.inf, math.nan
    op = bd.stacklstm_beam_create(1, 6, V, 2, 8, dt)
    got = out(1, 6)
    bd.stacklstm_beam_lse(op, z, got)
    g = got[0].tolist()
    assert g[:4] == [math.inf, math.inf, math.inf, -math.inf] and math.isnan(g[4]) and math.isfinite(g[5])


# ------------------------------------------------------------------ layer norm
def test_norm_of_the_most_rows():
    """2^31 - 1 rows: the last one and a step from it pass 31 bits."""
    R = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    op = bd.stacklstm_norm_create(R, 1, FP)
    x, beta = torch.ones(R, 1, device="cuda"), torch.full((1,), 3.0, device="cuda")
    y, mean, rstd = torch.zeros(R, 1, device="cuda"), torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
    bd.stacklstm_norm_forward(op, x, None, beta, 1.0, y, mean, rstd)
    bd.stacklstm_op_status(op)
    for t, want in ((y, 3.0), (mean, 1.0), (rstd, 1.0)):  # a row of one is its mean
        lo, hi = torch.aminmax(t)
        assert lo == want and hi == want
    y.fill_(0.0)
    y[-3:] = 1.0  # dy of the last rows alone, so that their sum is exact
    dx, dg, db = torch.full((R, 1), math.nan, device="cuda"), out(1), out(1)
    bd.stacklstm_norm_backward(op, y, x, None, mean, rstd, dx, dg, db)
    bd.stacklstm_op_status(op)
    lo, hi = torch.aminmax(dx)
    assert lo == 0 and hi == 0 and dg.item() == 0 and db.item() == 3


@TYPES
@pytest.mark.parametrize("R,N", [(12000, 40), (20000, 33), (3000, 1024), (900, 4096), (2000, 1025), (1300, 4099)])
def test_norm_of_more_rows_than_run_at_once(dt, R, N):
    """Every kernel's loop over rows, the wide one's too."""
    base.test_norm(dt, R, N)


# ------------------------------------------------------------------ fp32 numbers as parts
def one_a_row(rng, R, n, values):
    """[R, n] with one value a row, in different columns while there are as many."""
    a = np.zeros((R, n), np.float32)
    a[np.arange(R), rng.permutation(np.resize(rng.permutation(n), R))] = values
    return a


def odd(rng, bits, *s):
    """Numbers in [1, 2) of so many significant bits, the last one set."""
    return (1 + (2 * rng.integers(0, 2 ** (bits - 2), s) + 1) / 2 ** (bits - 1)).astype(np.float32)


# Products of 24 significant bits are exact in fp32, and so is every sum of their partial products:
# a part or a partial product that were left out would show. (significant bits of the factors; a bf16
# factor has 8 at most)
EXACT = pytest.mark.parametrize("bits", [(24, 1), (1, 24), (12, 12), (16, 8), (8, 16)])


def factor(rng, bits, *s):
    return 2.0 ** rng.integers(-3, 4, s) if bits == 1 else odd(rng, bits, *s)


@EXACT
@pytest.mark.parametrize("R,K,N", [(5, 70, 33), (64, 200, 100), (130, 75, 300)])
def test_linear_forward_takes_every_bit(bits, R, K, N):
    rng = np.random.default_rng(R + K + sum(bits))
    x, W = one_a_row(rng, R, K, factor(rng, bits[0], R)), np.float32(factor(rng, bits[1], N, K))
    op = bd.stacklstm_linear_create(R, K, N, FP)
    y = out(R, N)
    bd.stacklstm_linear_forward(op, up(x), up(W), None, None, y)
    assert np.array_equal(y.double().cpu().numpy(), x.astype(np.float64) @ W.T.astype(np.float64))


@TYPES
@EXACT
@pytest.mark.parametrize("R,K,N", [(20, 70, 33), (60, 75, 200), (290, 140, 300)])
def test_linear_backward_takes_every_bit(dt, bits, R, K, N):
    """dz is in three parts, x and W of fp32 too."""
    if dt == BF and bits[1] > 8:
        pytest.skip("not a bf16 number")
    rng = np.random.default_rng(R + K + sum(bits))
    dy = one_a_row(rng, R, N, factor(rng, bits[0], R))  # (no column of it has two values: R <= N)
    x, W = np.float32(factor(rng, bits[1], R, K)), np.float32(factor(rng, bits[1], N, K))
    op = bd.stacklstm_linear_create(R, K, N, dt)
    dx, dW, db = out(R, K), out(N, K), out(N)
    bd.stacklstm_linear_backward(op, up(dy), up(x, tdt(dt)), up(W, tdt(dt)), None, None, dx, dW, db)
    dy = dy.astype(np.float64)
    assert np.array_equal(dx.double().cpu().numpy(), dy @ W.astype(np.float64))
    assert np.array_equal(dW.double().cpu().numpy(), dy.T @ x.astype(np.float64))
    assert np.array_equal(db.double().cpu().numpy(), dy.sum(0))


# ------------------------------------------------------------------ more than 2^32 elements
def test_norm_offsets_beyond_32_bits():
    """The first and the last rows of 2^32 elements and more."""
    N = 1024
    R = (1 << 32) // N + 5
    x = torch.empty(R, N, dtype=torch.bfloat16, device="cuda").normal_()
    dy, dx = torch.zeros(R, N, device="cuda"), torch.full((R, N), math.nan, device="cuda")
    dy[-3:].normal_()
    y, mean, rstd, dg, db = torch.zeros_like(x), out(R), out(R), out(N), out(N)
    op = bd.stacklstm_norm_create(R, N, BF)
    bd.stacklstm_norm_forward(op, x, None, None, 1e-5, y, mean, rstd)
    bd.stacklstm_norm_backward(op, dy, x, None, mean, rstd, dx, dg, db)
    ends = torch.tensor([0, 1, R - 3, R - 2, R - 1], device="cuda")
    at = lambda t: base.f64(t[ends])
    wy, wm, wr = ol.norm_forward(at(x), None, None, 1e-5)
    # bounds as for smaller tensors, with |x| < 8 and 1 / 2 < rstd < 2 in these rows
    n = 2 * base.U * (N + 16)
    base.within(at(mean), wm, n * 8, "mean")
    base.within(at(rstd), wr, 2 * n * 17 * wr, "rstd")
    base.within(at(y), wy, 40 * n * (1 + np.abs(wy)) + 2.0 ** -8 * np.abs(wy), "y")
    wdx, wdg, wdb = ol.norm_backward(at(dy), at(x), None, at(mean), at(rstd))
    base.within(at(dx), wdx, 40 * n * (1 + np.abs(at(dy)).max()), "dx")
    base.within(base.f64(dg), wdg, 2.0 ** -20 * np.abs(at(dy) * 8).sum(0), "dgamma")
    base.within(base.f64(db), wdb, 2.0 ** -20 * np.abs(at(dy)).sum(0), "dbeta")
    assert not dx[:-3].any()


@TYPES
def test_linear_offsets_beyond_32_bits(dt):
    K, N = 64, 32003
    R = (1 << 32) // N + 7
    rng = np.random.default_rng(0)
    W, Wd = base.rounded(rng, dt, N, K, scale=1 / 8)
    xd = torch.empty(R, K, device="cuda").normal_().to(tdt(dt))
    op = bd.stacklstm_linear_create(R, K, N, dt)
    y = torch.zeros(R, N, dtype=tdt(dt), device="cuda")
    bd.stacklstm_linear_forward(op, xd, Wd, None, None, y)
    bd.stacklstm_op_status(op)
    ends = torch.tensor([0, 1, R - 3, R - 2, R - 1], device="cuda")
    x = base.f64(xd[ends])
    want = x @ W.T
    base.within(y[ends], want, 2 * base.U * (K + 16) * (np.abs(x) @ np.abs(W).T) + base.out_tol(dt, want), "y")
    assert y.count_nonzero(1).ge(N // 2).all()  # every row is written
    del y
    dy = torch.zeros(R, N, device="cuda")
    dy[-3:].normal_()
    dx, dW, db = torch.full((R, K), math.nan, device="cuda"), out(N, K), out(N)
    bd.stacklstm_linear_backward(op, dy, xd, Wd, None, None, dx, dW, db)
    bd.stacklstm_op_status(op)
    d = base.f64(dy[-3:])
    wx, wW, wb, _ = ol.linear_backward(d, x[-3:], W, None, None, "none")
    base.within(dx[-3:], wx, 2 * base.U * (N + 16) * (np.abs(d) @ np.abs(W)) + 4 * base.U * np.abs(wx), "dx")
    # (zeros add nothing: sums of three terms, in parts)
    base.within(dW, wW, 2.0 ** -19 * (np.abs(d).T @ np.abs(x[-3:])), "dW")
    base.within(db, wb, 2.0 ** -20 * np.abs(d).sum(0), "dbias")
    assert not dx[:-3].any()


@TYPES
@pytest.mark.parametrize("R,K,N", [(20, 70, 33), (130, 75, 300), (300, 136, 264)])
def test_linear_infinities_and_nan_stay_where_they_enter(dt, R, K, N):
    rng = np.random.default_rng(R)
    x, W, dy = base.rounded(rng, dt, R, K)[1], base.rounded(rng, dt, N, K)[1], up(rng.normal(size=(R, N)))
    x[3, 5], x[R - 1, K - 1], W[N - 1, 2], dy[7, 11] = math.inf, math.nan, -math.inf, math.nan
    op = bd.stacklstm_linear_create(R, K, N, dt)
    y, dx, dW, db = out(R, N, dtype=tdt(dt)), out(R, K), out(N, K), out(N)
    bd.stacklstm_linear_forward(op, x, W, None, None, y)
    bd.stacklstm_linear_backward(op, dy, x, W, None, None, dx, dW, db)
    bd.stacklstm_op_status(op)

    def only(t, rows, cols):
        bad = torch.zeros(t.shape, dtype=torch.bool, device="cuda")
        bad[rows] = True
        bad[..., cols] = True
        assert torch.equal(~t.isfinite(), bad)

    only(y, [3, R - 1], [N - 1])
    only(dx, [7], [2])
    only(dW, [11], [5, K - 1])
    assert (~db.isfinite()).nonzero().flatten().tolist() == [11]
