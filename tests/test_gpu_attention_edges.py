"""Calls of the attention, the log probabilities, the dropout and the attentive layers at the ends of what they take:
late warps, long memories, shifted logits, large scores, padding. Tolerances as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention as at
from paper_1904_03409_gb300 import binding as bd
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
    leaves less than 2^-7 of it) and the second rounded by up to 2^-8 of that, leave out 2^-15; of each tile of 64 states eight additions
    cut, each by less than 2^-23 of the sum so far (which is at most the sum of magnitudes)."""
    c = Case(BF, B, T, S, nh, nk, D)
    want, _, w = at.attend(*c.x, c.q_len, c.kv_len, float(c.scale))
    of = np.arange(nh) * nk // nh
    zmag = float(c.scale) * np.einsum("tbhd,sbhd->bhts", np.abs(c.x[0]), np.abs(c.x[1])[:, :, of])
    rel = 2 * (2 * U * (D + 8) + 4 * U) * zmag.max(3) + 4 * U * (S + 16) + 2.0 ** -20  # of a weight, as in Case.check
    wv = np.einsum("bhts,sbhd->tbhd", w, np.abs(c.x[2])[:, :, of])
    tol = (2 * rel.transpose(2, 0, 1)[..., None] + 2.0 ** -15 + 8 * 2.0 ** -23 * (S / 64 + 1)) * wv
    _, y, _, _ = c.forward(c.handle(), False)
    within(c.back(y, nh), want, tol * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(want), "y")
