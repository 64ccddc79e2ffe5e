"""A model on top of one StackLSTM: its outputs normalised, a hidden layer with a residual, scores
over V classes (labelled transitions, or words); training from a teacher's top logits and
decoding with a beam. Every computation is the library's (layer norm, linear, distillation
and beam calls of include/stacklstm.h); torch holds the tensors, draws the initial weights
and looks embeddings and per-class ops up.

    a      = norm(y)                                 y: the step outputs (tops) of the StackLSTM
    h      = gelu(a W1^T + b1) + a
    logits = h W2^T + b2
"""
from __future__ import annotations

import math

from . import binding as bd


def _raise_first(checks):
    """Every handle's status read (and so cleared), the first error raised."""
    errors = []
    for status, handle in checks:
        try:
            status(handle)
        except bd.StackLSTMError as e:
            errors.append(e)
    if errors:
        raise errors[0]


class OutputLayers:
    """The layers' weights and handles for up to ``rows`` tops of H units and V classes. Calls run on
    torch's current stream, whichever it is (a call on another one than the last waits, on the
    host, for what the layers did there)."""

    def __init__(self, rows: int, H: int, V: int, k: int, dtype: int = bd.SL_BF16, device: int = 0, seed: int = 0):
        import torch
        self.rows, self.H, self.V, self.k, self.dtype, self.device = rows, H, V, k, dtype, device
        dev = torch.device("cuda", device)
        dt = torch.bfloat16 if dtype == bd.SL_BF16 else torch.float32
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g) / math.sqrt(s[-1])).to(dev).to(dt)
        f = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
        t = lambda *s: torch.empty(*s, dtype=dt, device=dev)
        z = lambda *s: torch.zeros(*s, dtype=torch.float32, device=dev)
        self.params = dict(gamma=z(H) + 1, beta=z(H), W1=w(H, H), b1=z(H), W2=w(V, H), b2=z(V))
        self.grads = {n: f(*p.shape) for n, p in self.params.items()}
        self.norm = bd.stacklstm_norm_create(rows, H, dtype, device)
        self.hidden = bd.stacklstm_linear_create(rows, H, H, dtype, bd.SL_ACT_GELU, device)
        self.scores = bd.stacklstm_linear_create(rows, H, V, dtype, bd.SL_ACT_NONE, device)
        self.teacher = bd.stacklstm_distill_create(rows, V, k, dtype, device)
        self.a, self.pre, self.h, self.logits = t(rows, H), t(rows, H), t(rows, H), t(rows, V)
        self.mean, self.rstd, self.loss_rows, self.dlogits = f(rows), f(rows), f(rows), f(rows, V)
        self.dh, self.da, self.dy = f(rows, H), f(rows, H), f(rows, H)

    def _on_current_stream(self):
        import torch
        stream = torch.cuda.current_stream(self.device).cuda_stream
        for op in (self.norm, self.hidden, self.scores, self.teacher):
            if op.stream != stream:
                bd.stacklstm_op_set_stream(op, stream)

    def forward(self, y):
        """Logits of the tops y [r, H] (r up to ``rows``); what the backward needs is kept."""
        self._on_current_stream()
        r, p = y.shape[0], self.params
        bd.stacklstm_norm_forward(self.norm, y, p["gamma"], p["beta"], 1e-5, self.a[:r], self.mean[:r], self.rstd[:r])
        bd.stacklstm_linear_forward(self.hidden, self.a[:r], p["W1"], p["b1"], self.a[:r], self.h[:r], self.pre[:r])
        bd.stacklstm_linear_forward(self.scores, self.h[:r], p["W2"], p["b2"], None, self.logits[:r])
        return self.logits[:r]

    def learn(self, y, t_idx, t_logit, gold, tau=2.0, alpha=0.5):
        """Forward of the tops y [r, H], loss rows [r] against the teacher's k best (and the gold
        classes), the layers' gradients (``grads``) and the tops' gradient dy [r, H]."""
        r, p, g = y.shape[0], self.params, self.grads
        logits = self.forward(y)
        bd.stacklstm_distill_run(self.teacher, logits, t_idx, t_logit, gold, tau, alpha, 1.0 / max(r, 1), self.loss_rows[:r],
                                 self.dlogits[:r])
        bd.stacklstm_linear_backward(self.scores, self.dlogits[:r], self.h[:r], p["W2"], None, None, self.dh[:r], g["W2"], g["b2"])
        # the residual's gradient is dh itself
        bd.stacklstm_linear_backward(self.hidden, self.dh[:r], self.a[:r], p["W1"], self.pre[:r], self.dh[:r], self.da[:r], g["W1"],
                                     g["b1"])
        bd.stacklstm_norm_backward(self.norm, self.da[:r], y, p["gamma"], self.mean[:r], self.rstd[:r], self.dy[:r], g["gamma"],
                                   g["beta"])
        return self.loss_rows[:r], self.dy[:r]

    def status(self):
        _raise_first([(bd.stacklstm_op_status, op) for op in (self.norm, self.hidden, self.scores, self.teacher)])

    def destroy(self):
        for op in (self.norm, self.hidden, self.scores, self.teacher):
            op.destroy()


def train_step(hd, ins: dict, out: dict, layers: OutputLayers, t_idx, t_logit, gold, tau=2.0, alpha=0.5):
    """One training step of a StackLSTM (handle ``hd``, tensors as in ``runner``) under ``layers``:
    forward, loss against the teacher, backward. t_idx, t_logit [T B, k], gold [T B]; returns the
    loss rows; the gradients are in ``layers.grads`` and ``out``. ``hd`` may be on a stream of its
    own: the step comes after the current stream's work and before what follows on it."""
    import torch
    T, B, H = hd.T, hd.B, hd.H
    cur = torch.cuda.current_stream(hd.device)
    own = cur  # the StackLSTM's
    if hd.stream != cur.cuda_stream:
        own = torch.cuda.ExternalStream(hd.stream, hd.device) if hd.stream else torch.cuda.default_stream(hd.device)

    def order(first, then):
        if first is not then:
            then.wait_stream(first)

    order(cur, own)
    bd.stacklstm_forward(hd, ins["x"], ins["ops"], ins["h0"], ins["c0"], ins["W"], ins["bias"], None, None, out["p_final"], None,
                         None, out["y"])
    order(own, cur)
    loss, dy = layers.learn(out["y"].view(T * B, H), t_idx, t_logit, gold, tau, alpha)
    order(cur, own)
    bd.stacklstm_backward(hd, None, dy.view(T, B, H), out["dx"], out["dh0"], out["dc0"], out["dW"], out["dbias"])
    order(own, cur)
    return loss


def beam_decode(layers: OutputLayers, W, bias, emb, ops, h0, c0, K: int, steps: int, end: int = -1):
    """The K best sequences of up to ``steps`` classes for each of the B sentences whose stacks start
    at h0, c0 [B, H]. Class v pushes, pops or holds (ops [V] int8) with the input emb[v] (emb
    [V, I]); a pop of an empty stack is no candidate; class ``end`` ends a sequence. W, bias: the
    StackLSTM's. Returns (scores [B, K], classes [B, K, steps], -1 after an end), best first; where
    there are fewer than K sequences, -inf and -1."""
    import torch
    B, H = h0.shape
    V, I = emb.shape
    N, S, dt, dev = B * K, steps + 1, h0.dtype, h0.device
    f = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device=dev)
    t = lambda *s: torch.empty(*s, dtype=dt, device=dev)
    search = bd.stacklstm_beam_create(B, K, V, S, H, layers.dtype, layers.device)
    cell = bd.stacklstm_create(1, N, I, H, layers.dtype, layers.device)
    bd.stacklstm_set_async(cell, True)
    try:
        h, c, p = [t(S, N, H), t(S, N, H)], [f(S, N, H), f(S, N, H)], [torch.zeros(N, dtype=torch.int32, device=dev), i32(N)]
        top_h, top_c = h0.repeat_interleave(K, 0).contiguous(), c0.repeat_interleave(K, 0).contiguous()
        h[0][0], c[0][0] = top_h, top_c
        score = [torch.full((B, K), -math.inf, device=dev), f(B, K)]
        score[0][:, 0] = 0.0  # the first step expands one hypothesis a sentence
        lse, parent, token = f(B, K), i32(B, K), i32(B, K)
        done = torch.zeros(B, K, dtype=torch.uint8, device=dev)
        cell_h, cell_c, push = t(2, N, H), f(2, N, H), torch.ones(1, N, dtype=torch.int8, device=dev)
        p_cell = i32(N)
        history = torch.full((B, K, steps), -1, dtype=torch.int64, device=dev)
        pops = ops < 0
        for s in range(steps):
            logits = layers.forward(top_h)
            logits.masked_fill_((p[0] == 0)[:, None] & pops[None], -math.inf)
            logits = logits.view(B, K, V)
            bd.stacklstm_beam_lse(search, logits, lse)
            bd.stacklstm_beam_select(search, logits, lse, score[0], done, score[1], parent, token)
            bd.stacklstm_beam_reorder(search, parent, p[0], h[0], c[0], p[1], h[1], c[1], top_h, top_c)
            for pair in (h, c, p, score):
                pair.reverse()
            # the sequences' own bookkeeping: what each row comes from and whether it has ended
            from_row = parent.clamp_min(0).long()
            history = history.gather(1, from_row[..., None].expand_as(history)).contiguous()
            history.masked_fill_((parent < 0)[..., None], -1)  # candidates ran out: no sequence
            history[:, :, s] = token.long()
            done = done.gather(1, from_row)
            done |= ((token == end) & (token >= 0)).to(torch.uint8)
            cls = token.clamp_min(0).view(N).long()
            step_ops = torch.where(token.view(N) < 0, torch.zeros_like(ops[cls]), ops[cls]).contiguous()
            # the cell on the tops of all rows; what it gives is pushed where the class pushes
            bd.stacklstm_forward(cell, emb[cls].view(1, N, I), push, top_h, top_c, W, bias, cell_h, cell_c, p_cell)
            bd.stacklstm_beam_push(search, step_ops, cell_h[1], cell_c[1], p[0], h[0], c[0], top_h, top_c)
        _raise_first([(bd.stacklstm_status, cell)] +
                     [(bd.stacklstm_op_status, op) for op in (layers.norm, layers.hidden, layers.scores, search)])
        return score[0], history
    finally:
        search.destroy()
        cell.destroy()
