"""The output layers together on a StackLSTM: a training step's loss and gradients against the
fp64 oracles composed, and a beam search against one that recomputes every hypothesis from
its whole sequence in fp64."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import output_layers as ol
from paper_1904_03409_gb300 import binding as bd
from paper_1904_03409_gb300 import output_layers as om
from paper_1904_03409_gb300 import runner, workloads as wl

pytestmark = pytest.mark.gpu


def np64(d):
    return {k: v.double().cpu().numpy() for k, v in d.items()}


def layers_forward(p, y):
    a, m, r = ol.norm_forward(y, p["gamma"], p["beta"], 1e-5)
    h, pre = ol.linear_forward(a, p["W1"], p["b1"], a, "gelu")
    return ol.linear_forward(h, p["W2"], p["b2"], None, "none")[0], (a, m, r, pre, h)


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-4), ("bf16", 6e-2)])
def test_train_step(dtype, tol):
    # tolerances as those of the StackLSTM's own gradients (fp32: sums of fp32 terms through T
    # steps; bf16: three layers of activations rounded to 2^-9 each before the recurrence)
    T, B, H, V, k = 9, 12, 24, 37, 4
    w = wl.make_workload("model", T=T, B=B, I=16, H=H, dtype=dtype, seed=3, ops_kind="random_walk", probs=(0.5, 0.3, 0.2),
                         bias_scale=0.2, h0_scale=0.5)
    dt = bd.SL_BF16 if dtype == "bf16" else bd.SL_FP32
    rng = np.random.default_rng(4)
    R = T * B
    idx = rng.integers(-1, V, (R, k)).astype(np.int32)
    tl, gold = rng.normal(size=(R, k)).astype(np.float32), rng.integers(-1, V, R).astype(np.int32)
    hd = bd.stacklstm_create(T, B, 16, H, dt)
    layers = om.OutputLayers(R, H, V, k, dt, seed=7)
    ins, out = runner.upload(w), runner.alloc_outputs(w)
    up = lambda a: torch.from_numpy(a).cuda()
    loss = om.train_step(hd, ins, out, layers, up(idx), up(tl), up(gold))
    layers.status()
    bd.stacklstm_status(hd)
    ref = oracle.run(w.x, w.ops, w.h0, w.c0, w.W, w.bias, d_top_h=None, dy=None)
    p = np64(layers.params)
    y = ref["y"].reshape(R, H)
    logits, (a, m, r, pre, h) = layers_forward(p, y)
    want, d = ol.distill(logits, idx, tl, gold, 2.0, 0.5, 1.0 / R)
    dh, dW2, db2, _ = ol.linear_backward(d, h, p["W2"], None, None, "none")
    da, dW1, db1, _ = ol.linear_backward(dh, a, p["W1"], pre, dh, "gelu")
    dy, dg, dbt = ol.norm_backward(da, y, p["gamma"], m, r)
    full = oracle.run(w.x, w.ops, w.h0, w.c0, w.W, w.bias, dy=dy.reshape(T, B, H))

    def near(got, ref, what):
        err = np.abs(got.double().cpu().numpy() - ref).max()
        assert err <= tol * max(1e-30, np.abs(ref).max()), (what, err, np.abs(ref).max())

    near(loss, want, "loss")
    for n, g in (("W2", dW2), ("b2", db2), ("W1", dW1), ("b1", db1), ("gamma", dg), ("beta", dbt)):
        near(layers.grads[n], g, n)
    for n in ("dx", "dh0", "dc0", "dW", "dbias"):
        near(out[n], full[n], n)
    hd.destroy()
    layers.destroy()


def sequence_state(W, bias, emb, ops, h0, c0, seq):
    """Top (h, c) and depth after a sequence of classes, from the definition of the stack."""
    stack = [(h0, c0)]
    H = h0.size
    for v in seq:
        h, c = stack[-1]
        z = np.concatenate([emb[v], h]) @ W + bias
        i, f, g, o = (z[j * H:(j + 1) * H] for j in range(4))
        sg = lambda a: 1 / (1 + np.exp(-a))
        c2 = sg(f) * c + sg(i) * np.tanh(g)
        if ops[v] > 0:
            stack.append((sg(o) * np.tanh(c2), c2))
        elif ops[v] < 0:
            stack.pop()
    return stack[-1][0], len(stack) - 1


def test_beam_decode():
    """fp32; the scores of neighbouring hypotheses differ by far more than fp32 rounding."""
    B, K, V, H, I, steps, end = 3, 4, 9, 16, 8, 6, 8
    rng = np.random.default_rng(11)
    f = lambda *s, sc=1.0: (sc * rng.normal(size=s)).astype(np.float32)
    W, bias, emb = f(I + H, 4 * H, sc=0.4), f(4 * H, sc=0.2), f(V, I)
    h0, c0 = np.tanh(f(B, H)), f(B, H)
    ops = np.array([1, 1, 1, -1, -1, 0, 0, 1, 0], np.int8)
    layers = om.OutputLayers(B * K, H, V, 1, bd.SL_FP32, seed=5)
    layers.params["W2"] *= 3.0
    up = lambda a: torch.from_numpy(a).cuda()
    score, seqs = om.beam_decode(layers, up(W), up(bias), up(emb), up(ops), up(h0), up(c0), K, steps, end)
    layers.status()
    p = np64(layers.params)
    for b in range(B):
        beam = [(0.0, [], False)]
        for _ in range(steps):
            found = []
            for n, (s, seq, done) in enumerate(beam):
                if done:
                    found.append((s, n * V, seq, True))
                    continue
                h, depth = sequence_state(W.astype(np.float64), bias.astype(np.float64), emb.astype(np.float64), ops,
                                          h0[b].astype(np.float64), c0[b].astype(np.float64), seq)
                z = layers_forward(p, h[None])[0][0]
                if depth == 0:
                    z = np.where(ops < 0, -np.inf, z)
                lp = z - ol.lse(z[None, None])[0, 0]
                found += [(s + lp[v], n * V + v, seq + [v], v == end) for v in range(V) if lp[v] > -math.inf]
            found.sort(key=lambda e: (-e[0], e[1]))
            beam = [(s, seq, done) for s, _, seq, done in found[:K]]
        for j, (s, seq, _) in enumerate(beam):
            assert seqs[b, j].tolist() == seq + [-1] * (steps - len(seq))
            assert abs(float(score[b, j]) - s) <= 1e-4
    layers.destroy()
