"""Calls of the attention, the log probabilities, the dropout and the attentive layers at the ends of what they take:
late warps, long memories, shifted logits, large scores, padding. Tolerances as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as at
from paper_1904_03409_gb300 import binding as bd
from paper_1904_03409_gb300 import output_layers as om
import test_gpu_attention as tga
from test_gpu_attention import BF, FP, TYPES, U, Case, empty, tdt, within

pytestmark = pytest.mark.gpu


@TYPES
@pytest.mark.parametrize("D", [40, 64, 128])
def test_many_short_sentences_with_broken_tiles(dt, D):
    """Thousands of items of one to four tiles, whole and broken ones in turn, so that the warp that clears behind a
    sentence's end often has loads of several items behind it: no wait runs out, the same bits every time."""
    B, T, S, nh = 90, 140, 256, 4
    g = torch.Generator(device="cuda").manual_seed(D)
    r = lambda n: torch.randn(n, B, nh * D, device="cuda", generator=g).to(tdt(dt))
    q, k, v, dy = r(T), r(S), r(S), r(T).float()
    q_len = torch.randint(0, T + 1, (B,), device="cuda", generator=g).int()
    kv_len = (64 * torch.randint(0, 5, (B,), device="cuda", generator=g) - torch.randint(0, 2, (B,), device="cuda", generator=g)).clamp_min(0).int()
    op = bd.stacklstm_attend_create(T, S, B, nh, nh, D, dt)
    first = None
    for _ in range(5):
        y0, y, lse, ctx = empty(*q.shape, dtype=tdt(dt)), empty(*q.shape, dtype=tdt(dt)), empty(T, B, nh), empty(*q.shape)
        bd.stacklstm_attend_forward(op, q, k, v, q_len, kv_len, D ** -0.5, y0)
        bd.stacklstm_attend_forward(op, q, k, v, q_len, kv_len, D ** -0.5, y, lse, ctx)
        grads = [empty(n, B, nh * D) for n in (T, S, S)]
        bd.stacklstm_attend_backward(op, dy, q, k, v, q_len, kv_len, D ** -0.5, lse, ctx, *grads)
        bd.stacklstm_op_status(op)
        out = [y0, y, lse, ctx, *grads]
        assert not any(torch.isnan(t).any() for t in out)
        assert first is None or all(torch.equal(a, b) for a, b in zip(out, first))
        first = first or out


@pytest.mark.parametrize("B,T,S,nh,nk,D", [(1, 8, 40, 5, 5, 40), (2, 64, 65, 2, 2, 63), (1, 65, 128, 1, 1, 128), (1, 129, 129, 2, 1, 72),
                                           (1, 127, 300, 4, 2, 100), (1, 2, 1100, 6, 2, 32), (2, 5, 3000, 4, 1, 64)])
def test_a_bf16_result_alone_keeps_its_weights(B, T, S, nh, nk, D):
    """Without ctx as with it: y is what the weights in fp32 give, rounded once. Two bf16 parts of a weight, the first cut (which
    leaves less than 2^-7 of it) and the second rounded by up to 2^-8 of that, leave out 2^-15; of each tile of 64 states eight MMAs cut
    what they add: over 2^20 states of one sign y lost 0.9 %, 2^-23.8 of the sum an MMA, here 2^-23 of the sum of magnitudes."""
    c = Case(BF, B, T, S, nh, nk, D)
    want, _, w = at.attend(*c.x, c.q_len, c.kv_len, float(c.scale))
    of = np.arange(nh) * nk // nh
    zmag = float(c.scale) * np.einsum("tbhd,sbhd->bhts", np.abs(c.x[0]), np.abs(c.x[1])[:, :, of])
    rel = 2 * (2 * U * (D + 8) + 4 * U) * zmag.max(3) + 4 * U * (S + 16) + 2.0 ** -20  # of a weight, as in Case.check
    wv = np.einsum("bhts,sbhd->tbhd", w, np.abs(c.x[2])[:, :, of])
    tol = (2 * rel.transpose(2, 0, 1)[..., None] + 2.0 ** -15 + 8 * 2.0 ** -23 * (S / 64 + 1)) * wv
    _, y, _, _ = c.forward(c.handle(), False)
    within(c.back(y, nh), want, tol * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want), "y")


def long_reference(q, k, v, kv_len, scale, nk):
    """y of q [T, B, nk D] and the sum of magnitudes sum w |v| in fp64, some heads at a time, with the bound on a weight's error
    (as in Case.check)."""
    T, B, S, D = q.shape[0], q.shape[1], k.shape[0], k.shape[2] // nk
    y, mag, rel = (torch.empty(T, B, nk, d, device="cuda", dtype=torch.float64) for d in (D, D, 1))
    step = max(1, 2 ** 28 // (S * D))
    for b in range(B):
        n = S if kv_len is None else int(kv_len[b])
        for h in range(0, nk, step):
            cut = lambda x, n: x[:n, b].view(n, nk, D)[:, h:h + step].double()
            qq, kk, vv = cut(q, T), cut(k, n), cut(v, n)
            w = torch.softmax(scale * torch.einsum("tnd,snd->nts", qq, kk), -1)
            zmag = scale * torch.einsum("tnd,snd->nts", qq.abs(), kk.abs()).amax(2)
            y[:, b, h:h + step] = torch.einsum("nts,snd->tnd", w, vv)
            mag[:, b, h:h + step] = torch.einsum("nts,snd->tnd", w, vv.abs())
            rel[:, b, h:h + step, 0] = (2 * (2 * U * (D + 8) + 4 * U) * zmag + 4 * U * 4096 + 2.0 ** -20).t()
    return y, mag, rel


@pytest.mark.parametrize("B,T,S,nk,D,ragged", [(1, 1, 9000, 320, 16, False), (2, 2, 8300, 160, 24, True), (1, 3, 5000, 320, 72, False),
                                               (1, 2, 300000, 2, 24, False), (3, 130, 4200, 110, 8, True)])
def test_memories_of_several_sums(B, T, S, nk, D, ragged):
    """More than 4096 states to an item, in several sums that are joined in fp32: scores that grow along the states, so that
    each sum has a base of its own; whole and broken ends; a few long sentences, split as well. Cuts of 8 MMAs a tile,
    2^-23 of the sum of magnitudes each as above, and 64 tiles at most, weights in two parts, and an fp32 sum (4 u a term) of the runs."""
    g = torch.Generator(device="cuda").manual_seed(S)
    r = lambda n: torch.randn(n, B, nk * D, device="cuda", generator=g)
    grow = torch.linspace(0, 20, S, device="cuda")[:, None, None]
    q, k, v = r(T).abs().bfloat16(), (0.5 * r(S) + grow / D ** 0.5).bfloat16(), r(S).bfloat16()
    kv_len = torch.tensor([S, 4097, 64][:B], dtype=torch.int32, device="cuda") if ragged else None
    op = bd.stacklstm_attend_create(T, S, B, nk, nk, D, BF)
    y = empty(*q.shape, dtype=torch.bfloat16)
    scale = float(np.float32(D ** -0.5))
    bd.stacklstm_attend_forward(op, q, k, v, None, kv_len, scale, y)
    bd.stacklstm_op_status(op)
    want, mag, rel = long_reference(q, k, v, kv_len, scale, nk)
    tol = (2 * rel + 2.0 ** -15 + 512 * 2.0 ** -23 + 8 * U * (S / 4096 + 33)) * mag
    within(y.view_as(want), want.cpu().numpy(), (tol * (1 + 2.0 ** -7) + 2.0 ** -8 * want.abs()).cpu().numpy(), "y")


def test_the_longest_memory():
    """2^20 states of values of one sign, not split (320 heads): no bias from additions that cut. Of a result's mean relative error
    rounding to bf16 leaves 2^-8 / sqrt(3 n) of n results whose sizes spread over an octave (four of those), the cuts of one sum of
    4096 states 2^-14 at most."""
    S, nk, D = 1 << 20, 320, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(1, 1, nk * D, device="cuda", generator=g).bfloat16()
    k = torch.randn(S, 1, nk * D, device="cuda", generator=g, dtype=torch.bfloat16)
    v = torch.rand(S, 1, nk * D, device="cuda", generator=g, dtype=torch.bfloat16)
    v += 1
    v *= torch.exp2(torch.rand(nk * D, device="cuda", generator=g)).bfloat16()
    op = bd.stacklstm_attend_create(1, S, 1, nk, nk, D, BF)
    y = empty(1, 1, nk * D, dtype=torch.bfloat16)
    bd.stacklstm_attend_forward(op, q, k, v, None, None, D ** -0.5, y)
    bd.stacklstm_op_status(op)
    want, mag, rel = long_reference(q, k, v, None, D ** -0.5, nk)
    off = y.view_as(want).double() / want - 1
    assert abs(float(off.mean())) <= 2.0 ** -14 + 4 * 2.0 ** -8 / (3 * nk * D) ** 0.5
    tol = 2 * rel + 2.0 ** -15 + 2.0 ** -14 + 8 * U * 289
    assert bool((off.abs() <= tol * (1 + 2.0 ** -7) + 2.0 ** -8).all())


@TYPES
@pytest.mark.parametrize("R,V,k", [(5, 7, 2), (9, 83, 5), (40, 432, 3), (6, 2500, 4), (160, 2500, 4), (3, 32003, 2), (90, 32003, 2), (2, 70001, 3),
                                   (40, 70001, 1), (2, 300007, 0)])
@pytest.mark.parametrize("kind", [300, 3000, -1e5, "rows of -1e9", "rows of the lowest"])
def test_the_logits_gradient_does_not_depend_on_a_shift(dt, R, V, k, kind):
    """Logits far from 0, and finite rows masked throughout. Errors, relative to p times what it is multiplied by: the sum of
    exponentials of up to 64 terms a thread and its joins, 96 u; exponents, by 8 u of them (of their mean in the sum) and
    of ln f, which is what half a step of lse leaves, 21 at most; two exponentials, 2^-21 each; the weights' sum, 2 u a
    term. Nothing grows with the logits."""
    rng = np.random.default_rng(R + V)
    z = 3 * rng.normal(size=(R, V)) + (kind if not isinstance(kind, str) else 0.0)
    if isinstance(kind, str):
        z[::2] = -1e9 if kind.endswith("9") else float(torch.finfo(tdt(dt)).min)
    zd = torch.from_numpy(z).to(tdt(dt)).cuda()
    z = zd.double().cpu().numpy()
    target = rng.integers(-1, V, R).astype(np.int32)
    op = bd.stacklstm_logprob_create(R, V, k, dt)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    logp, ent, lse, idx, top = empty(R), empty(R), empty(R), empty(R, k, dtype=torch.int32), empty(R, k)
    bd.stacklstm_logprob_forward(op, zd, up(target), logp, ent, lse, idx if k else None, top if k else None)
    g, h, gt = (rng.normal(size=s).astype(np.float32) for s in (R, R, (R, k)))
    x = z.max(1, keepdims=True) - z
    e = np.exp(-x)
    p = e / e.sum(1, keepdims=True)
    mean = (p * np.minimum(x, 200)).sum(1, keepdims=True)
    rest = np.minimum(21, U * np.abs(lse.double().cpu().numpy()))[:, None]
    rel = U * (min(V, 64) + 32) + 2.0 ** -20 + 8 * U * (np.minimum(x, 200) + mean + rest + 4) + 2 * U * (k + 2)
    _, we, _, wi, _ = at.logprob(z, target, k)
    hits = np.zeros_like(z)
    for r in range(R):
        for c in [target[r], *wi[r]]:
            if c >= 0:
                hits[r, c] = np.abs(g[r]) + np.abs(gt[r]).sum()
    d = empty(R, V)
    for a in ((g, None, gt), (g, h, gt), (None, h, None)):
        bd.stacklstm_logprob_backward(op, zd, up(target), ent, lse, idx if k else None, up(a[0]) if a[0] is not None else None,
                                      up(a[1]) if a[1] is not None else None, up(gt) if k and a[2] is not None else None, d)
        bd.stacklstm_op_status(op)
        want = at.logprob_backward(z, target, wi, *a)
        mag = sum(np.abs(v).reshape(R, -1).sum(1, keepdims=True) for v in (a[0], a[2]) if v is not None) if a[0] is not None else 0.0
        if a[1] is not None:  # (the entropy, of its own sums, enters here as well)
            mag = mag + np.abs(h)[:, None] * (x + np.abs(we)[:, None] + np.log(V) + 1)
        within(d, want, p * np.where(p > 0, mag, 0) * 2 * rel + 2 * U * (k + 4) * hits + 1e-37, "dlogits")


@TYPES
@pytest.mark.parametrize("offset", [0, 300, 3200, -3200])
@pytest.mark.parametrize("B,T,S,nh,nk,D", [(2, 40, 1300, 2, 2, 64), (1, 2, 5000, 6, 2, 128), (3, 30, 90, 4, 4, 40)])
def test_results_of_large_scores(dt, offset, B, T, S, nh, nk, D):
    """Scores around `offset` that fp32 holds exactly (products of whole numbers of few bits), in splits and whole: y in fp32 as exact as
    around 0. Of a weight, independent of one another: its exponent's rounding, at most 11 u in each of two operations, the
    exponential 2^-21, its sum and the division 4 u, cut sums of 12 products of parts 12 x 1.7e-8, a split's weight the same
    again: sqrt(2 (2 x 0.66^2 + 0.48^2 + 0.24^2) + 0.2^2) = 1.5e-6 at most. lse: by half a step and 2^-20."""
    g = torch.Generator(device="cuda").manual_seed(S + D)
    r = lambda n, h: torch.randint(-1, 2, (n, B, h, D), device="cuda", generator=g).float()
    q, k, v = r(T, nh), r(S, nk), torch.randn(S, B, nk, D, device="cuda", generator=g)
    q[..., 0], k[..., 0] = 25.0, offset / 6.25  # (of a quarter: `offset` itself)
    q, k, v = (t.to(tdt(dt)).flatten(2) for t in (q, k, v))
    kv_len = torch.tensor([S, S // 2, 70][:B], device="cuda").int()
    h = lambda x: x.double().view(x.shape[0], B, nk, -1, D)
    see = torch.arange(S, device="cuda")[None] < kv_len[:, None]
    z = (0.25 * torch.einsum("tbngd,sbnxd->bngts", h(q), h(k))).masked_fill(~see.view(B, 1, 1, 1, S), -float("inf"))
    want = torch.einsum("bngts,sbnxd->tbngd", torch.softmax(z, -1), h(v))
    op = bd.stacklstm_attend_create(T, S, B, nh, nk, D, dt)
    y, lse, ctx = empty(*q.shape, dtype=tdt(dt)), empty(T, B, nh), empty(*q.shape)
    bd.stacklstm_attend_forward(op, q, k, v, None, kv_len, 0.25, y, lse, ctx)
    bd.stacklstm_op_status(op)
    assert float((ctx.double().view(want.shape) - want).norm()) <= 1.5e-6 * float(want.norm())
    wl = torch.logsumexp(z, -1).permute(3, 0, 1, 2).reshape(T, B, nh)
    assert bool(((lse.double() - wl).abs() <= U * wl.abs() + 2.0 ** -20).all())


@TYPES
@pytest.mark.parametrize("offset", [0, 300, 3200, -3200])
@pytest.mark.parametrize("B,T,S,nh,nk,D", [(3, 119, 300, 8, 2, 40), (1, 700, 130, 2, 1, 112), (2, 40, 1300, 2, 2, 64), (20, 130, 60, 8, 8, 24)])
def test_gradients_of_large_scores(dt, offset, B, T, S, nh, nk, D):
    """Scores around `offset` that fp32 holds exactly (products of whole numbers of few bits): gradients as a whole as exact as those
    of scores around 0. Of a weight, which the bound of test_gradients_keep_32_bits_over_many_states leaves without
    lse's rounding: sqrt(0.24^2 + 2 x 0.66^2 + 0.48^2 + 0.41^2) = 1.2e-6 of it at most. One at a time the same bits."""
    g = torch.Generator(device="cuda").manual_seed(S + D)
    r = lambda n, h, m: torch.randint(-m, m + 1, (n, B, h, D), device="cuda", generator=g).float()
    q, k = r(T, nh, 1), r(S, nk, 1)
    q[..., 0], k[..., 0] = 25.0, offset / 6.25  # (of a quarter: `offset` itself)
    v, dy = torch.randn(S, B, nk, D, device="cuda", generator=g), torch.randn(T, B, nh, D, device="cuda", generator=g)
    q, k, v = (t.to(tdt(dt)).flatten(2) for t in (q, k, v))
    dy, scale = dy.flatten(2), 0.25
    q_len, kv_len = torch.tensor([T, T // 2, T][:B] + [T] * (B - 3), device="cuda").int(), torch.tensor([S, S, S // 3][:B] + [S] * (B - 3), device="cuda").int()
    h = lambda x: x.double().view(x.shape[0], B, nk, -1, D)
    see = torch.arange(S, device="cuda")[None] < kv_len[:, None]
    use = (torch.arange(T, device="cuda")[:, None] < q_len[None]).view(T, B, 1, 1, 1)
    z = (scale * torch.einsum("tbngd,sbnxd->bngts", h(q), h(k))).masked_fill(~see.view(B, 1, 1, 1, S), -float("inf"))
    w = torch.softmax(z, -1)
    dw = torch.einsum("tbngd,sbnxd->bngts", h(dy) * use, h(v))
    dz = scale * w * (dw - (w * dw).sum(-1, keepdim=True))
    want = (torch.einsum("bngts,sbnxd->tbngd", dz, h(k)), torch.einsum("bngts,tbngd->sbnd", dz, h(q)), torch.einsum("bngts,tbngd->sbnd", w, h(dy) * use))
    op = bd.stacklstm_attend_create(T, S, B, nh, nk, D, dt)
    y, lse, ctx = empty(*q.shape, dtype=tdt(dt)), empty(T, B, nh), empty(*q.shape)
    bd.stacklstm_attend_forward(op, q, k, v, q_len, kv_len, scale, y, lse, ctx)
    grads = [empty(n, B, c * D) for n, c in ((T, nh), (S, nk), (S, nk))]
    bd.stacklstm_attend_backward(op, dy, q, k, v, q_len, kv_len, scale, lse, ctx, *grads)
    bd.stacklstm_op_status(op)
    for name, a, b in zip(("dq", "dk", "dv"), grads, want):
        a = a.double().view(b.shape)
        if name == "dq":  # (column 0 is the states' common one, a sum of dz: nothing but its rounding)
            a, b = a[..., 1:], b[..., 1:]
        assert float((a - b).norm()) <= 1.2e-6 * float(b.norm()), name
    for i in range(3):
        one = [torch.full_like(t, float("nan")) if j == i else None for j, t in enumerate(grads)]
        bd.stacklstm_attend_backward(op, dy, q, k, v, q_len, kv_len, scale, lse, ctx, *one)
        assert torch.equal(one[i], grads[i])
    bd.stacklstm_op_status(op)


@TYPES
def test_gradients_of_sharp_weights(dt, monkeypatch):
    """z in the hundreds with the backward: weights down to e^-300 and below, of which those under 2^-126 (and parts of numbers
    under it) are 0 in fp32. A gradient's 40 terms are such a number times |dy . v| <= 64 x 4 x 4, |q| <= 30 and the scale
    of 1 at most: 2^-126 x 40 x 1024 x 30 < 2^-105."""
    monkeypatch.setattr(tga, "within", lambda got, want, tol, what="": within(got, want, tol + 2.0 ** -105, what))
    Case(dt, 2, 20, 300, 2, 2, 64, scale=1.0, sharp=6.0).check()


@pytest.mark.parametrize("S,nk,D", [(1, 1, 16), (1, 2, 21), (300, 1, 64), (70, 2, 100)])
@pytest.mark.parametrize("scale", [1.0, 40.0])
def test_a_single_state_has_weight_1(S, nk, D, scale):
    """Whatever its score is: y = v and dv the sum of dy, finite also at the largest numbers (three parts of a number, of sums that
    may cut: 4 u), dq = dk = 0; sentences of one state among others."""
    T, B = 3, 3
    big = float(torch.finfo(torch.float32).max)
    g = torch.Generator(device="cuda").manual_seed(D)
    r = lambda n, h: torch.randn(n, B, h * D, device="cuda", generator=g)
    q, k, v, dy = r(T, nk), r(S, nk), r(S, nk), r(T, nk)
    v[..., ::3], v[..., 4] = big, -big
    dy[1:] = 0  # (a sum of one)
    dy[0, :, 1::2], dy[0, :, 2] = big, 2.0 ** -126
    kv_len = torch.tensor([1, S, 1], device="cuda").int()
    if S > 1:  # (a mean of the largest numbers is its own concern)
        v[:, 1], dy[:, 1] = r(S, nk)[:, 1], r(T, nk)[:, 1]
    op = bd.stacklstm_attend_create(T, S, B, nk, nk, D, FP)
    y, lse, grads = empty(T, B, nk * D), empty(T, B, nk), [empty(n, B, nk * D) for n in (T, S, S)]
    bd.stacklstm_attend_forward(op, q, k, v, None, kv_len, scale, y, lse)
    bd.stacklstm_attend_backward(op, dy, q, k, v, None, kv_len, scale, lse, y, *grads)
    bd.stacklstm_op_status(op)
    for b in (0, 2):
        for got, want in ((y[:, b], v[:1, b].expand(T, -1)), (grads[2][:1, b], dy[:1, b])):
            assert torch.isfinite(got).all() and bool(((got - want).abs().double() <= 4 * U * want.abs().double()).all())
        assert not grads[0][:, b].any() and not grads[1][:, b].any() and not grads[2][1:, b].any()
    z = scale * (q[:, 0].double() * k[:1, 0].double()).view(T, nk, D).sum(-1)
    assert bool(((lse[:, 0].double() - z).abs() <= 2 * U * scale * (D + 9) * (q[:, 0].abs() * k[:1, 0].abs()).view(T, nk, D).sum(-1)).all())


@TYPES
def test_rows_behind_a_sentences_end_have_no_part_in_the_objective(dt):
    """A constant weight of the entropy, and anything in dlogp: the same gradients as with zeros there."""
    T, B, S, H, E, V, heads = 7, 4, 9, 24, 16, 13, 2
    rng = np.random.default_rng(3)
    up = lambda a, t=None: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t or torch.float32)
    q_len = up([7, 3, 1, 0], torch.int32)
    inside = torch.arange(T, device="cuda")[:, None] < q_len[None]
    y, mem = up(rng.normal(size=(T * B, H)), tdt(dt)), up(rng.normal(size=(S, B, E)), tdt(dt))
    target, g = up(rng.integers(0, V, T * B), torch.int32), up(rng.normal(size=T * B)).view(T, B)
    out = []
    for dlogp, dent in ((torch.where(inside, g, float("nan")), torch.full((T, B), 0.1, device="cuda")),
                        (torch.where(inside, g, 0.0), torch.where(inside, 0.1, 0.0))):
        layers = om.AttentiveLayers(T, B, S, H, E, V, heads, p=0.2, dtype=dt, seed=5)
        layers.memory(mem)
        _, _, dy, dstates = layers.learn(y, target, dlogp.reshape(-1), dent.reshape(-1), q_len)
        layers.status()
        out.append([t.clone() for t in (dy, dstates, *layers.grads.values())])
        assert torch.isfinite(dy).all() and not dy.view(T, B, H)[~inside].any()
        layers.destroy()
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("rows,mask_rows", [(1500000000, 1000000000), (2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 2)])
def test_dropout_of_rows_and_mask_rows_beyond_31_bits(rows, mask_rows):
    op = bd.stacklstm_dropout_create(rows, 1, BF)
    x = torch.ones(rows, 1, device="cuda", dtype=torch.bfloat16)
    bd.stacklstm_dropout_forward(op, x, None, 0.5, 5, None, mask_rows, x)
    bd.stacklstm_op_status(op)
    keep = at.keep(min(mask_rows, 1000), 1, 0, 0.5, 5, 0)
    assert ((x[: len(keep), 0].double().cpu().numpy() == 2) == keep).all()
    if mask_rows == 1:
        assert bool((x == x[0]).all())
    else:
        assert torch.equal(x[mask_rows:], x[: rows - mask_rows]) and bool(((x == 0) | (x == 2)).all())


def test_sizes_that_the_attentive_layers_refuse():
    """Sentences other than those whose states they look at (4 rows were taken for 4 sentences of one hypothesis where they were 2
    of two), tops of fewer or more steps, states of another width."""
    B, S, H, E, V, I = 4, 5, 16, 8, 7, 8
    layers = om.AttentiveLayers(2, B, S, H, E, V, 2, beam=2, dtype=FP)
    x = lambda *s: torch.randn(*s, device="cuda")
    for shape in ((S + 1, B, E), (S, B + 1, E), (S, 2 * B, E // 2), (S, B * E)):
        with pytest.raises(ValueError):
            layers.memory(x(*shape))
    layers.memory(x(S, B, E))
    ops = torch.ones(V, device="cuda", dtype=torch.int8)
    for n, K in ((2, 2), (B, 3)):
        with pytest.raises(ValueError):
            om.beam_decode(layers, x(I + H, 4 * H), x(4 * H), x(V, I), ops, x(n, H), x(n, H), K, 3)
    score, _ = om.beam_decode(layers, x(I + H, 4 * H), x(4 * H), x(V, I), ops, x(B, H), x(B, H), 2, 3)
    assert torch.isfinite(score).all()
    grads = [g.fill_(7.0) for g in layers.grads.values()]
    zero = torch.zeros(2 * B, device="cuda")
    for rows in (2 * B - 1, B, 2 * B + 1):
        with pytest.raises(ValueError):
            layers.learn(x(rows, H), zero.int(), zero, zero)
    assert all(bool((g == 7.0).all()) for g in grads) and int(layers.step) == 0
    layers.status()
    layers.destroy()
