"""Models on top of one StackLSTM: its outputs normalised, a hidden layer with a residual (or attention
over an encoder's states), scores over V classes (labelled transitions, or words); training from a
teacher's top logits, or as a policy, and decoding with a beam. Every computation is the library's
(layer norm, linear, distillation, attention, dropout, log-probability and beam calls of
include/stacklstm.h); torch holds the tensors, draws the initial weights and looks embeddings and
per-class ops up.

    OutputLayers:     a      = norm(y)                                 y: the step outputs (tops) of the StackLSTM
                      h      = gelu(a W1^T + b1) + a
                      logits = h W2^T + b2
    AttentiveLayers:  u      = attention of a Wq^T over the states' Wk^T and Wv^T
                      h      = dropout(u Wo^T + bo) + a                one mask a sentence for all of its steps
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

    def _ops(self):
        return self.norm, self.hidden, self.scores, self.teacher

    def _on_current_stream(self):
        import torch
        stream = torch.cuda.current_stream(self.device).cuda_stream
        for op in self._ops():
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

    def decoders(self):
        """The handles that a forward uses."""
        return self.norm, self.hidden, self.scores

    def status(self):
        _raise_first([(bd.stacklstm_op_status, op) for op in self._ops()])

    def destroy(self):
        for op in self._ops():
            op.destroy()


class AttentiveLayers:
    """Layers that look at an encoder's states: weights and handles for B sentences of up to T tops of H units
    and S states of E units, ``heads`` heads (``kv_heads`` of them in the states) and V classes, and for beams of
    up to ``beam`` hypotheses. Calls run on torch's current stream, as OutputLayers' do."""

    def __init__(self, T: int, B: int, S: int, H: int, E: int, V: int, heads: int, kv_heads: int = 0, p: float = 0.1, k: int = 0,
                 beam: int = 1, dtype: int = bd.SL_BF16, device: int = 0, seed: int = 0):
        import torch
        kv_heads = kv_heads or heads
        if H % heads:
            raise ValueError("H must be a multiple of the heads")
        D = H // heads
        rows, most = T * B, max(T, beam) * B
        self.T, self.B, self.S, self.H, self.E, self.V, self.k, self.p, self.beam = T, B, S, H, E, V, k, p, beam
        self.rows, self.dtype, self.device, self.seed, self.scale = rows, dtype, device, seed, D ** -0.5
        dev = torch.device("cuda", device)
        dt = torch.bfloat16 if dtype == bd.SL_BF16 else torch.float32
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g) / math.sqrt(s[-1])).to(dev).to(dt)
        f = lambda *s: torch.empty(*s, dtype=torch.float32, device=dev)
        t = lambda *s: torch.empty(*s, dtype=dt, device=dev)
        z = lambda *s: torch.zeros(*s, dtype=torch.float32, device=dev)
        C = kv_heads * D
        self.params = dict(gamma=z(H) + 1, beta=z(H), Wq=w(H, H), Wk=w(C, E), Wv=w(C, E), Wo=w(H, H), bo=z(H), W2=w(V, H), b2=z(V))
        self.grads = {n: f(*p.shape) for n, p in self.params.items()}
        self.step = torch.zeros(1, dtype=torch.int64, device=dev)  # of training: each has masks of its own
        lin = lambda R, K, N: bd.stacklstm_linear_create(R, K, N, dtype, bd.SL_ACT_NONE, device)
        self.norm = bd.stacklstm_norm_create(most, H, dtype, device)
        self.query, self.keys, self.values, self.mix, self.scores = (lin(most, H, H), lin(S * B, E, C), lin(S * B, E, C), lin(most, H, H),
                                                                    lin(most, H, V))
        self.attend = bd.stacklstm_attend_create(T, S, B, heads, kv_heads, D, dtype, bd.SL_TIME_MAJOR, bd.SL_TIME_MAJOR, device)
        self.look = bd.stacklstm_attend_create(beam, S, B, heads, kv_heads, D, dtype, bd.SL_BATCH_MAJOR, bd.SL_TIME_MAJOR, device)
        self.drop = bd.stacklstm_dropout_create(rows, H, dtype, device)
        self.policy = bd.stacklstm_logprob_create(rows, V, k, dtype, device)
        self.a, self.q, self.u, self.o, self.h, self.logits = t(most, H), t(most, H), t(most, H), t(most, H), t(most, H), t(most, V)
        self.kk, self.vv, self.kv_len, self.s = t(S, B, C), t(S, B, C), None, 0
        self.mean, self.rstd = f(most), f(most)
        self.lse, self.ctx = f(T, B, heads), f(T, B, H) if dtype == bd.SL_BF16 else None
        self.logp, self.entropy, self.z = f(rows), f(rows), f(rows)
        self.top_idx, self.top_logp = (torch.empty(rows, k, dtype=torch.int32, device=dev), f(rows, k)) if k else (None, None)
        self.dlogits, self.dh, self.do, self.du, self.dq, self.da, self.dy = f(rows, V), f(rows, H), f(rows, H), f(T, B, H), f(T, B, H), f(rows, H), f(rows, H)
        self.dk, self.dv, self.dstates = f(S, B, C), f(S, B, C), f(S * B, E)

    def _ops(self):
        return (self.norm, self.query, self.keys, self.values, self.mix, self.scores, self.attend, self.look, self.drop, self.policy)

    def decoders(self):
        return self.norm, self.query, self.keys, self.values, self.mix, self.scores, self.look

    _on_current_stream = OutputLayers._on_current_stream

    def memory(self, states, kv_len=None):
        """The encoder's states [s, B, E] (s up to S; kv_len [B] int32 of them in each sentence, the others finite)
        that the following calls look at."""
        if states.dim() != 3 or states.shape[0] > self.S or states.shape[1:] != (self.B, self.E):
            raise ValueError("states must be [s, %d, %d] of at most %d states" % (self.B, self.E, self.S))
        self._on_current_stream()
        s = states.shape[0]
        flat, kv = states.reshape(s * self.B, self.E), (self.kk[:s].view(s * self.B, -1), self.vv[:s].view(s * self.B, -1))
        for op, name, to in ((self.keys, "Wk", kv[0]), (self.values, "Wv", kv[1])):
            bd.stacklstm_linear_forward(op, flat, self.params[name], None, None, to)
        self.states, self.kv_len, self.s = flat, kv_len, s

    def _have_memory(self):
        if not self.s:
            raise ValueError("memory() comes first: the states to look at")

    def _tops(self, y, train, attend):
        """a, q, what attend() makes of q (u), and u Wo^T + bo (train: without the residual a) of the tops y [r, H]."""
        r, p = y.shape[0], self.params
        bd.stacklstm_norm_forward(self.norm, y, p["gamma"], p["beta"], 1e-5, self.a[:r], self.mean[:r], self.rstd[:r])
        bd.stacklstm_linear_forward(self.query, self.a[:r], p["Wq"], None, None, self.q[:r])
        attend()
        bd.stacklstm_linear_forward(self.mix, self.u[:r], p["Wo"], p["bo"], None if train else self.a[:r], self.o[:r] if train else self.h[:r])

    def forward(self, y):
        """Logits of the tops y [B K, H] of K hypotheses of each sentence (no dropout)."""
        self._on_current_stream()
        self._have_memory()
        r = y.shape[0]
        K = r // self.B
        if K * self.B != r or K > self.beam:
            raise ValueError("y must have the same number of rows for each sentence, %d at most" % self.beam)
        at = lambda x: x[:r].view(self.B, K, self.H)
        self._tops(y, False, lambda: bd.stacklstm_attend_forward(self.look, at(self.q), self.kk[:self.s], self.vv[:self.s], None, self.kv_len,
                                                                 self.scale, at(self.u)))
        bd.stacklstm_linear_forward(self.scores, self.h[:r], self.params["W2"], self.params["b2"], None, self.logits[:r])
        return self.logits[:r]

    def learn(self, y, target, dlogp, dentropy, q_len=None):
        """Forward with dropout of the tops y [T B, H] (q_len [B] of them in each sentence, the others finite), and the
        gradients of the objective whose gradient with respect to each row's log probability of its target (-1: none) and
        entropy is dlogp, dentropy [T B] (whatever they are behind a sentence's end: those rows have no part in it): the
        layers' (``grads``), the tops' dy [T B, H] and the states' dstates [s B, E]. Returns (logp, entropy, dy, dstates)."""
        import torch
        if y.shape != (self.rows, self.H):
            raise ValueError("y must be [%d, %d]: the tops of every step of every sentence" % (self.rows, self.H))
        self._on_current_stream()
        self._have_memory()
        r, p, g, s = self.rows, self.params, self.grads, self.s
        T, B, H = self.T, self.B, self.H
        if q_len is not None:
            behind = (torch.arange(T, device=y.device)[:, None] >= q_len[None]).view(r)
            dlogp, dentropy = (None if d is None else d.masked_fill(behind, 0.0) for d in (dlogp, dentropy))
        at = lambda x: x[:r].view(T, B, H)
        kk, vv, lens = self.kk[:s], self.vv[:s], (q_len, self.kv_len)
        self._tops(y, True, lambda: bd.stacklstm_attend_forward(self.attend, at(self.q), kk, vv, *lens, self.scale, at(self.u), self.lse, self.ctx))
        # one mask a sentence: row t B + b takes mask row b
        bd.stacklstm_dropout_forward(self.drop, self.o[:r], self.a[:r], self.p, self.seed, self.step, B, self.h[:r])
        bd.stacklstm_linear_forward(self.scores, self.h[:r], p["W2"], p["b2"], None, self.logits[:r])
        logits = self.logits[:r]
        bd.stacklstm_logprob_forward(self.policy, logits, target, self.logp, self.entropy, self.z, self.top_idx, self.top_logp)
        bd.stacklstm_logprob_backward(self.policy, logits, target, self.entropy, self.z, None, dlogp, dentropy, None, self.dlogits)
        bd.stacklstm_linear_backward(self.scores, self.dlogits, self.h[:r], p["W2"], None, None, self.dh, g["W2"], g["b2"])
        bd.stacklstm_dropout_backward(self.drop, self.dh, None, self.p, self.seed, self.step, B, self.do)
        bd.stacklstm_linear_backward(self.mix, self.do, self.u[:r], p["Wo"], None, None, self.du.view(r, H), g["Wo"], g["bo"])
        bd.stacklstm_attend_backward(self.attend, self.du, at(self.q), kk, vv, *lens, self.scale, self.lse,
                                     at(self.u) if self.ctx is None else self.ctx, self.dq, self.dk[:s], self.dv[:s])
        # the residual's gradient is dh itself
        bd.stacklstm_linear_backward(self.query, self.dq.view(r, H), self.a[:r], p["Wq"], None, self.dh, self.da, g["Wq"])
        dstates = self.dstates[:s * B]
        bd.stacklstm_linear_backward(self.keys, self.dk[:s].view(s * B, -1), self.states, p["Wk"], None, None, dstates, g["Wk"])
        bd.stacklstm_linear_backward(self.values, self.dv[:s].view(s * B, -1), self.states, p["Wv"], None, dstates, dstates, g["Wv"])
        bd.stacklstm_norm_backward(self.norm, self.da, y, p["gamma"], self.mean[:r], self.rstd[:r], self.dy, g["gamma"], g["beta"])
        self.step += 1
        return self.logp, self.entropy, self.dy, dstates

    def status(self):
        _raise_first([(bd.stacklstm_op_status, op) for op in self._ops()])

    def destroy(self):
        for op in self._ops():
            op.destroy()


def train_step(hd, ins: dict, out: dict, layers: OutputLayers, t_idx, t_logit, gold, tau=2.0, alpha=0.5):
    """One training step of a StackLSTM (handle ``hd``, tensors as in ``runner``) under ``layers``:
    forward, loss against the teacher, backward. t_idx, t_logit [T B, k], gold [T B]; returns the
    loss rows; the gradients are in ``layers.grads`` and ``out``. ``hd`` may be on a stream of its
    own: the step comes after the current stream's work and before what follows on it."""
    return _stack_step(hd, ins, out, lambda y: layers.learn(y, t_idx, t_logit, gold, tau, alpha)[::-1])


def policy_step(hd, ins: dict, out: dict, layers: AttentiveLayers, target, dlogp, dentropy, q_len=None):
    """One training step of a StackLSTM under ``layers`` as a policy over its classes (their ``memory`` set):
    target, dlogp, dentropy [T B] as in ``AttentiveLayers.learn`` (for a step along the gradient of
    sum(weight logp + c entropy) over each sentence's q_len rows: -weight and -c). Returns (logp, entropy, dstates); the gradients are in
    ``layers.grads`` and ``out``. Streams as in ``train_step``."""
    def learn(y):
        logp, entropy, dy, dstates = layers.learn(y, target, dlogp, dentropy, q_len)
        return dy, (logp, entropy, dstates)
    return _stack_step(hd, ins, out, learn)


def _stack_step(hd, ins: dict, out: dict, learn):
    """Forward of the StackLSTM, learn(tops [T B, H]) -> (their gradient, result), its backward."""
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
    dy, result = learn(out["y"].view(T * B, H))
    order(cur, own)
    bd.stacklstm_backward(hd, None, dy.view(T, B, H), out["dx"], out["dh0"], out["dc0"], out["dW"], out["dbias"])
    order(own, cur)
    return result


def beam_decode(layers, W, bias, emb, ops, h0, c0, K: int, steps: int, end: int = -1):
    """The K best sequences of up to ``steps`` classes for each of the B sentences whose stacks start
    at h0, c0 [B, H] under ``layers``: OutputLayers, or AttentiveLayers of B sentences whose ``memory``
    holds their states. Class v pushes, pops or holds (ops [V] int8) with the input emb[v] (emb
    [V, I]); a pop of an empty stack is no candidate; class ``end`` ends a sequence. W, bias: the
    StackLSTM's. Returns (scores [B, K], classes [B, K, steps], -1 after an end), best first; where
    there are fewer than K sequences, -inf and -1."""
    import torch
    B, H = h0.shape
    V, I = emb.shape
    if isinstance(layers, AttentiveLayers) and (layers.B != B or K > layers.beam):
        raise ValueError("the layers look at the states of %d sentences, for beams of at most %d" % (layers.B, layers.beam))
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
                     [(bd.stacklstm_op_status, op) for op in (*layers.decoders(), search)])
        return score[0], history
    finally:
        search.destroy()
        cell.destroy()
