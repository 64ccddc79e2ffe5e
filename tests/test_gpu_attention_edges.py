"""Calls of the attention, the log probabilities, the dropout and the attentive layers at the ends of what they take:
late warps, long memories, shifted logits, large scores, padding. Tolerances as in test_gpu_attention.py."""
import pytest
import torch

from paper_1904_03409_gb300 import binding as bd
from test_gpu_attention import BF, FP, TYPES, empty, tdt

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
